// Attention of one new token of each sequence over a paged cache:
// sifar_paged_attention. gfx950 (MI355X) only.
//
// Every key and value that is there has to be read once, and 4 operations per element of
// them for each query head that shares it: bound by HBM bytes, for short sequences by
// the launch and the chain length -> page -> keys -> values. So keys and values go from
// memory straight into the registers that the matrix instructions read, and the query
// heads of one cache head (up to 16) are the columns of one tile, so that the cache is
// read once for all of them.
//
// With S = K Q^T (positions x heads), P = exp2(S - m) and O = V^T P (elements x heads):
//  - K's tile is read as it lies: a lane holds 16 bytes of one position's row.
//  - S's tile leaves in each lane 4 positions of one head, which are as they stand
//    the summands that a lane holds of P in V^T P: positions need no order, as long as
//    V's rows come in the same one. Nothing crosses lanes but the maximum.
//  - A lane loads 16 bytes of each of its positions' values, 16 lanes a whole row; for
//    16-bit elements a byte permute per word turns them into columns.
//  - The running maximum m, the sums and O stay in registers, all for the head of
//    the lane's column, so rescaling O is a product in each lane, done only when some
//    head's maximum has grown.
// P is split into two 16-bit elements (what the first leaves goes into the second), so
// weights are good to 2^-17 and the output's one rounding is its last; the second
// product costs matrix time that the bytes leave free.
// Infinite values would meet the second elements' zeros and signs: where a wave's sums are
// not finite, it takes its tiles once more and gives those values a product of their own.
// (Looking costs 0.1 us a call, 1 x 33 in a graph 4.7 and 4.8; with infinities in every
// sequence 64 ragged ones take 394 us instead of 208.)
//
// A workgroup takes one cache head of one sequence, or a chunk of its positions where that
// leaves too few workgroups or too uneven ones; its four waves take every fourth tile and
// join in LDS. Chunks' sums go to the workspace, not yet divided, and a second launch joins
// them.
//
// Measured, bf16, heads of 128: 1 x 131072 (32 heads on 8) 91.5 us a call, 5.9 TB/s, which is
// what loads in this pattern reach that compute nothing; 64 x 4096 (64 on 8) 190 us, 5.7; 64
// sequences of 1 to 8192 (1056 MB) 227 us, 4.6 (the rest are chunks of unequal length, the
// last of which leave CUs idle); 1 x 33 in a graph 4.8 us. Left out, the matrix products and the
// softmax change none of the long ones by a percent; nor do coalesced keys, or a third
// less or more workgroups a CU.
#include <hip/hip_runtime.h>

#include "attend_plan.h"
#include "paged.h"
#include "rows.h"
#include "sifar_kernels.h"
#include "tiles.h"

namespace sifar {
namespace {

constexpr int kThreads = kWaves * kRowWave;
constexpr float kLog2e = 0x1.715476p+0f, kLn2 = 0x1.62e430p-1f;
constexpr float kLowest = -0x1.fffffep127f;  // below every finite score
constexpr float kFar = 0x1p127f;  // times log2(e) still finite

struct AttendArgs {
    sifar_paged_attention_args a;
    DivU32 page;    // by page_size
    DivU32 splits;  // by the most chunks of a sequence
    int32_t group;  // query heads of a cache head
    int32_t reach;  // lengths are cut to this
    int32_t round;  // chunks are multiples of this, a power of two
    float unit;     // log2(e), or 1 where the scale or softcap leaves fp32 times it: then last
    int64_t at_outs;  // the chunks' outputs from the workspace's start, in floats
};

// Which positions a sequence has, and how long its chunks are.
struct Stretch {
    int first, count, chunk;
};
__device__ __forceinline__ Stretch stretch(const AttendArgs &n, int64_t t) {
    int length = n.a.lengths[t];
    length = length < 0 ? 0 : length > n.reach ? n.reach : length;
    Stretch s;
    s.first = n.a.window > 0 && length > n.a.window ? length - n.a.window : 0;
    s.count = length - s.first;
    s.chunk = chunk_of(
        static_cast<int>(div_u32(static_cast<uint32_t>(s.count) + n.splits.d - 1, n.splits)),
        n.round);
    return s;
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_of(float x) { return __builtin_amdgcn_logf(x); }

// tanh: its series where 1 - 2 / (e^2y + 1) would cancel (off by 2e-8 at 0.35).
__device__ __forceinline__ float tanh_of(float y) {
    const float a = __builtin_fabsf(y), z = y * y;
    float p = -0x1.226e36p-7f;  // -1382 / 155925
    p = __builtin_fmaf(p, z, 0x1.664f48p-6f);
    p = __builtin_fmaf(p, z, -0x1.ba1ba2p-5f);
    p = __builtin_fmaf(p, z, 0x1.111112p-3f);
    p = __builtin_fmaf(p, z, -0x1.555556p-2f);
    const float near = __builtin_fmaf(p * z, y, y);
    const float far =
        __builtin_copysignf(1.f - 2.f / (exp2_of(2.f * kLog2e * a) + 1.f), y);
    return a < 0.35f ? near : far;
}

template <int N>
using Words = uint32_t __attribute__((ext_vector_type(N)));

// Keys and values: ONCE, past the caches, where there are more of them than the caches keep
// until the next call.
template <class T, bool ONCE>
__device__ __forceinline__ T load_cache(const unsigned char *p) {
    const T *at = reinterpret_cast<const T *>(p);
    return ONCE ? __builtin_nontemporal_load(at) : *at;
}

// Four adjacent outputs.
template <int D>
__device__ __forceinline__ void store4(void *row, int64_t at, const F4 &f) {
    Stored<D> *p = static_cast<Stored<D> *>(row) + at;
    if constexpr (D == SIFAR_FP32) {
        *reinterpret_cast<F4 *>(p) = f;
    } else {
        typedef uint32_t U2 __attribute__((ext_vector_type(2)));
        *reinterpret_cast<U2 *>(p) = U2{pack16<D>(f[0], f[1]), pack16<D>(f[2], f[3])};
    }
}

// What a row's sum of weights l, relative to 2^m, makes of its output and of lse.
struct Close {
    float inverse, lse;
};
__device__ __forceinline__ Close close_row(const AttendArgs &n, int head, float m, float l) {
    if (n.a.sinks) {
        const float natural = n.a.sinks[head], two = natural * kLog2e;
        // one that has no place in base 2 keeps one at its end
        const float sink =
            natural < kLowest ? natural : __builtin_fminf(__builtin_fmaxf(two, kLowest), -kLowest);
        const float top = sink > m ? sink : m;
        const float scale = exp2_of(m - top);
        const float whole = l * scale + exp2_of(sink - top);
        return {whole == 0.f ? 0.f : scale / whole,
                sink >= m ? natural + log2_of(whole) * kLn2 : (top + log2_of(whole)) * kLn2};
    }
    return {l == 0.f ? 0.f : 1.f / l, (l == 0.f ? -__builtin_inff() : (m + log2_of(l)) * kLn2)};
}

// The lane's index, as a value of its own: what a loop's body derives from it is computed
// there, and not kept in registers around the loops inside, where keys, values and sums
// need them.
__device__ __forceinline__ int own_thread() {
    int i = threadIdx.x;
    asm volatile("" : "+v"(i));
    return i;
}

// What is infinite or NaN in a tile of 16-bit values, added to the sums and taken out of the
// tile. A weight's second element is often zero or of the other sign, and an infinity times
// it NaN: so those values meet the weights' signs alone, in a product of their own (1 where
// there is weight; zero and NaN as they are). Sums that they leave finite keep their bits.
template <int D, int SUBS, int MINE, int PANELS, int WORDS, int SUMS>
__device__ __forceinline__ void take_strange(const F4 (&x)[SUBS],
                                             uint32_t (&v)[MINE][PANELS][WORDS],
                                             F4 (&o)[SUMS]) {
    constexpr uint32_t kExponent = D == SIFAR_BF16 ? 0x7F80u : 0x7C00u;
    const auto strange = [](uint32_t w) {  // all bits of the halves whose exponent is full
        return ((w & kExponent) == kExponent ? 0xFFFFu : 0u) |
               ((w >> 16 & kExponent) == kExponent ? 0xFFFF0000u : 0u);
    };
    const auto sign = [](float w) { return w > 0.f ? 1.f : w; };
    Half<MINE / 2> s;
#pragma unroll
    for (int j = 0; j < MINE / 2; ++j)
        s.w[j] = pack16<D>(sign(x[j / 2][2 * (j & 1)]), sign(x[j / 2][2 * (j & 1) + 1]));
#pragma unroll
    for (int p = 0; p < PANELS; ++p)
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            Half<MINE / 2> even, odd;
#pragma unroll
            for (int j = 0; j < MINE / 2; ++j) {
                uint32_t &a = v[2 * j][p][i], &b = v[2 * j + 1][p][i];
                const uint32_t keep_a = ~strange(a), keep_b = ~strange(b);
                even.w[j] = __builtin_amdgcn_perm(b & ~keep_b, a & ~keep_a, 0x05040100u);
                odd.w[j] = __builtin_amdgcn_perm(b & ~keep_b, a & ~keep_a, 0x07060302u);
                a &= keep_a;
                b &= keep_b;
            }
            F4 &e = o[p * 2 * WORDS + 2 * i], &d = o[p * 2 * WORDS + 2 * i + 1];
            e = mma_half<D>(even, s, e);
            d = mma_half<D>(odd, s, d);
        }
}

// D: element type. DIM: 64, 128 or 256, head_dim or the next above it (PAD).
template <int D, int DIM, bool PAD, bool ONCE>
__global__ void __launch_bounds__(kThreads, held_by_a_cu(D, DIM, PAD))
attend_kernel(const AttendArgs n) {
    constexpr int SIZE = D == SIFAR_FP32 ? 4 : 2;
    constexpr int STEPS = DIM * SIZE / 64;          // of 64 bytes of a row of keys
    // positions: half as many where keys, values and O would not fit the registers
    constexpr int TILE = tile_of(D, DIM);
    constexpr int SUBS = TILE / 16;
    constexpr int MINE = TILE / 4;                  // positions whose values a lane loads
    // 16 lanes hold a row of values in panels, up to 16 bytes a lane each
    constexpr int BYTES = DIM * SIZE / 16 < 16 ? DIM * SIZE / 16 : 16;
    constexpr int EACH = BYTES / SIZE, WORDS = BYTES / 4;
    constexpr int PANELS = DIM / (16 * EACH);
    constexpr int ROW = DIM + 4;  // floats of a head's output in LDS, off the banks' period
    // fp16 weights are taken 2^14 times as large, which l's share undoes: small ones then
    // keep their bits. bf16 has fp32's exponents.
    constexpr float UP = D == SIFAR_FP16 ? 14.f : 0.f;

    constexpr int kPlaceBytes = kMaxChunk * 4, kOutBytes = kWaves * 16 * ROW * 4;
    __shared__ alignas(16) unsigned char lds[kPlaceBytes > kOutBytes ? kPlaceBytes : kOutBytes];
    __shared__ float top[kWaves][16], sum[kWaves][16];
    __shared__ uint32_t gone[kMaxChunk / 32];  // a bit for each position that is not there
    uint32_t *place = reinterpret_cast<uint32_t *>(lds);
    float *outs = reinterpret_cast<float *>(lds);

    const sifar_paged_attention_args &a = n.a;
    const int64_t t = blockIdx.z;
    const int piece = blockIdx.x, splits = gridDim.x;
    const int kv = blockIdx.y % a.kv_heads, tile16 = blockIdx.y / a.kv_heads;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int column = lane & 15, quarter = lane >> 4;
    const int heads = n.group - 16 * tile16 < 16 ? n.group - 16 * tile16 : 16;  // columns in use
    const int first_head = kv * n.group + 16 * tile16;
    const int fours = a.head_dim / 4;

    const Stretch s = stretch(n, t);
    const int from = piece * s.chunk;  // behind s.first
    const int count = s.count - from < s.chunk ? s.count - from : s.chunk;
    if (count <= 0) {  // the same for the workgroup
        if (splits > 1) return;  // not a chunk: the second launch knows
        for (int i = threadIdx.x; i < heads * fours; i += kThreads) {
            store4<D>(a.out, t * a.out_stride + static_cast<int64_t>(first_head) * a.head_dim +
                                 4 * i, F4{0.f, 0.f, 0.f, 0.f});
            if (a.lse && i < heads)
                a.lse[t * a.q_heads + first_head + i] =
                    close_row(n, first_head + i, kLowest, 0.f).lse;
        }
        return;
    }

    const int64_t head_at = static_cast<int64_t>(kv) * a.head_stride * SIZE;
    const unsigned char *k_cache = static_cast<const unsigned char *>(a.k_cache) + head_at;
    const unsigned char *v_cache = static_cast<const unsigned char *>(a.v_cache) + head_at;
    const int row_bytes = a.head_dim * SIZE;
    // The queries' operand: in registers, or, where keys, values and O leave no room for
    // it, in LDS, the same for all waves.
    constexpr bool SHARED = DIM > 64;
    __shared__ U4 q_lds[SHARED ? STEPS * kRowWave : 1];
    U4 q[STEPS];
    U4 k[SUBS][STEPS];
    uint32_t v[MINE][PANELS][WORDS];
    // Lanes behind the end of a head's row load its first bytes and drop them (times the
    // queries' zeros, what is not finite would count). The row ends in the second half.
    constexpr int SURE = !PAD ? STEPS : DIM > 64 ? STEPS / 2 : 0;
    const unsigned char *k_lane = k_cache + 16 * quarter, *k_end[STEPS];
    uint32_t keep[STEPS];
#pragma unroll
    for (int i = SURE; i < STEPS; ++i) {
        keep[i] = 64 * i + 16 * quarter < row_bytes ? ~0u : 0u;
        k_end[i] = k_cache + (keep[i] & (64 * i + 16 * quarter));
    }
    const unsigned char *v_lane[PANELS];
#pragma unroll
    for (int p = 0; p < PANELS; ++p)
        v_lane[p] = v_cache + (!PAD || (16 * p + column) * BYTES < row_bytes
                                   ? (16 * p + column) * BYTES
                                   : 0);
    const auto load_keys = [&](int tile) {
#pragma unroll
        for (int j = 0; j < SUBS; ++j) {
            const uint64_t at =
                static_cast<uint64_t>(place[tile * TILE + 16 * j + column]) * (8 * SIZE);
#pragma unroll
            for (int i = 0; i < STEPS; ++i)
                k[j][i] = load_cache<U4, ONCE>(i < SURE ? k_lane + at + 64 * i : k_end[i] + at);
        }
    };
    const auto load_values = [&](int tile) {
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
            const uint64_t at =
                static_cast<uint64_t>(place[tile * TILE + 16 * (j / 4) + 4 * quarter + (j & 3)]) *
                (8 * SIZE);
#pragma unroll
            for (int p = 0; p < PANELS; ++p) {
                const Words<WORDS> w = load_cache<Words<WORDS>, ONCE>(v_lane[p] + at);
#pragma unroll
                for (int i = 0; i < WORDS; ++i) v[j][p][i] = w[i];
            }
        }
    };

    const uint32_t page_eights = static_cast<uint32_t>(a.page_stride / 8);
    const uint32_t slot_eights = static_cast<uint32_t>(a.slot_stride / 8);
    // The queries' loads go out before the places', and are used behind them.
    {
        const unsigned char *row =
            static_cast<const unsigned char *>(a.q) +
            (t * a.q_stride +
             static_cast<int64_t>(first_head + (column < heads ? column : 0)) * a.head_dim) * SIZE;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int at = 64 * i + 16 * quarter;
            q[i] = *reinterpret_cast<const U4 *>(row + (!PAD || at < row_bytes ? at : 0));
        }
    }
    // Where positions lie, in eights of elements from the head's first; a position that is
    // not there gets the place of the first slot, which is, and its bit.
    const int tiles = (count + TILE - 1) / TILE;
    constexpr int EACH_LANE = kMaxChunk / kThreads;
    int pages[EACH_LANE];  // all loaded before one is used
    uint32_t slots[EACH_LANE];
#pragma unroll
    for (int j = 0; j < EACH_LANE; ++j) {
        const int i = j * kThreads + static_cast<int>(threadIdx.x);
        const uint32_t p = static_cast<uint32_t>(s.first + from + (i < count ? i : count - 1));
        const uint32_t nth = div_u32(p, n.page);
        slots[j] = p - nth * n.page.d;
        pages[j] = a.pages[t * a.pages_stride + nth];
    }
#pragma unroll
    for (int j = 0; j < EACH_LANE; ++j) {
        const int i = j * kThreads + static_cast<int>(threadIdx.x);
        const bool there = i < count &&
                           static_cast<uint32_t>(pages[j]) < static_cast<uint32_t>(a.num_pages);
        const uint64_t at = static_cast<uint64_t>(pages[j]) * page_eights +
                            static_cast<uint64_t>(slots[j]) * slot_eights;
        place[i] = there ? static_cast<uint32_t>(at) : 0u;
        const uint64_t missing = __builtin_amdgcn_ballot_w64(!there);
        if ((i & 31) == 0) gone[i / 32] = static_cast<uint32_t>(missing >> (i & 63));
    }
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const bool in = column < heads && (!PAD || 64 * i + 16 * quarter < row_bytes);
        q[i] &= in ? ~0u : 0u;
        if (SHARED && wave == 0) q_lds[i * kRowWave + lane] = q[i];
    }
    __syncthreads();

    float m = kLowest, l = 0.f;
    F4 o[PANELS * EACH];
#pragma unroll
    for (int i = 0; i < PANELS * EACH; ++i) o[i] = F4{0.f, 0.f, 0.f, 0.f};

    // A tile's part of the sums; with MORE the wave's next one is loaded on the way. (The
    // last one stands behind the loop: where its loads were left out by a branch inside,
    // the registers of values were reused too early, in fp32 heads of 256.)
    const auto take = [&](int tile, auto more, auto strange) {
        constexpr bool MORE = decltype(more)::value, STRANGE = decltype(strange)::value;
        if (SHARED) {
            asm volatile("" ::: "memory");  // loaded here, not kept from before the loop
#pragma unroll
            for (int i = 0; i < STEPS; ++i) q[i] = q_lds[i * kRowWave + lane];
        }
        uint32_t missing = __builtin_amdgcn_readfirstlane(gone[tile * TILE / 32]);
        if (TILE == 16) missing = missing >> (16 * (tile & 1)) & 0xFFFFu;
        // S: positions x heads
        F4 x[SUBS];
#pragma unroll
        for (int j = 0; j < SUBS; ++j) {
            x[j] = F4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                if (i >= SURE) k[j][i] &= keep[i];
                x[j] = mma<D>(k[j][i], q[i], x[j]);
            }
        }
        if constexpr (MORE) load_keys(tile + kWaves);

#pragma unroll
        for (int j = 0; j < SUBS; ++j) {
            if (a.softcap > 0.f) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    x[j][r] = a.softcap * n.unit * tanh_of(x[j][r] * a.scale / a.softcap);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) x[j][r] *= a.scale * n.unit;
            }
        }
        if (n.unit == 1.f) {
#pragma unroll
            for (int j = 0; j < SUBS; ++j) x[j] *= kLog2e;
        }
        if (missing) {
#pragma unroll
            for (int j = 0; j < MINE; ++j) {
                const bool not_there = missing >> (16 * (j / 4) + 4 * quarter + (j & 3)) & 1;
                x[j / 4][j & 3] = not_there ? -__builtin_inff() : x[j / 4][j & 3];
                // weight 0 times what the slot holds would be NaN if that is not finite
                const uint32_t keep = not_there ? 0u : ~0u;
#pragma unroll
                for (int p = 0; p < PANELS; ++p)
#pragma unroll
                    for (int w = 0; w < WORDS; ++w) v[j][p][w] &= keep;
            }
        }
        float high = x[0][0];
#pragma unroll
        for (int j = 0; j < SUBS; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) high = __builtin_fmaxf(high, x[j][r]);
        const auto up = [](Pair<float> p) { return __builtin_fmaxf(p.a, p.b); };
        high = up(pair<16>(high));
        high = up(pair<32>(high));
        high = __builtin_fmaxf(high, m);
        if (__builtin_amdgcn_ballot_w64(high > m)) {
            const float shrink = exp2_of(m - high);
            m = high;
            l *= shrink;
#pragma unroll
            for (int i = 0; i < PANELS * EACH; ++i) o[i] *= shrink;
        }
#pragma unroll
        for (int j = 0; j < SUBS; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[j][r] = exp2_of(x[j][r] - m + UP);
                l += x[j][r];
            }

        // O: elements x heads
        if constexpr (D == SIFAR_FP32) {
#pragma unroll
            for (int p = 0; p < PANELS; ++p)
#pragma unroll
                for (int i = 0; i < EACH; ++i)
#pragma unroll
                    for (int j = 0; j < MINE; ++j)
                        o[p * EACH + i] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                            __uint_as_float(v[j][p][i]), x[0][j], o[p * EACH + i], 0, 0, 0);
        } else {
            if constexpr (STRANGE) take_strange<D>(x, v, o);
            Half<MINE / 2> hi, lo;
#pragma unroll
            for (int j = 0; j < MINE / 2; ++j) {
                const Split w = split<D>(x[j / 2][2 * (j & 1)], x[j / 2][2 * (j & 1) + 1]);
                hi.w[j] = w.high;
                lo.w[j] = w.low;
            }
#pragma unroll
            for (int p = 0; p < PANELS; ++p)
#pragma unroll
                for (int i = 0; i < WORDS; ++i) {
                    Half<MINE / 2> even, odd;  // columns 2 i and 2 i + 1 of this lane's positions
#pragma unroll
                    for (int j = 0; j < MINE / 2; ++j) {
                        even.w[j] = __builtin_amdgcn_perm(v[2 * j + 1][p][i], v[2 * j][p][i],
                                                          0x05040100u);
                        odd.w[j] = __builtin_amdgcn_perm(v[2 * j + 1][p][i], v[2 * j][p][i],
                                                         0x07060302u);
                    }
                    F4 &e = o[p * EACH + 2 * i], &d = o[p * EACH + 2 * i + 1];
                    e = mma_half<D>(even, hi, e);
                    d = mma_half<D>(odd, hi, d);
                    e = mma_half<D>(even, lo, e);
                    d = mma_half<D>(odd, lo, d);
                }
        }
        if constexpr (MORE) load_values(tile + kWaves);
    };
    const auto take_all = [&](auto strange) {
        int tile = wave;
        load_keys(tile);
        load_values(tile);
        for (; tile + kWaves < tiles; tile += kWaves) take(tile, std::true_type{}, strange);
        take(tile, std::false_type{}, strange);
    };
    if (wave < tiles) {
        take_all(std::false_type{});
        // Values of 16 bits that are not finite need a product of their own: only where a sum
        // shows that there may be some are the tiles taken once more, with it.
        if constexpr (D != SIFAR_FP32) {
            F4 all = o[0];
#pragma unroll
            for (int i = 1; i < PANELS * EACH; ++i) all += o[i];
            const float any = __builtin_fabsf(all[0] + all[1] + (all[2] + all[3]));
            if (__builtin_amdgcn_ballot_w64(!(any < __builtin_inff()))) {
                asm volatile("" ::: "memory");  // loaded again, not kept
                m = kLowest;
                l = 0.f;
#pragma unroll
                for (int i = 0; i < PANELS * EACH; ++i) o[i] = F4{0.f, 0.f, 0.f, 0.f};
                take_all(std::true_type{});
            }
        }
    }

    // The waves' sums, joined relative to the largest of their maxima.
    const int thread = own_thread(), own_column = thread & 15, own_quarter = thread >> 4 & 3;
    const auto add = [](Pair<float> p) { return p.a + p.b; };
    l = add(pair<16>(l));
    l = add(pair<32>(l));
    if (own_quarter == 0) {
        top[wave][own_column] = m;
        sum[wave][own_column] = l;
    }
    __syncthreads();  // also: no wave reads places any more
    const int busy = count < kWaves * TILE ? (count + TILE - 1) / TILE : kWaves;  // had a tile
    if (wave < busy && own_column < heads) {
        float most_of_all = top[0][own_column];
        for (int w = 1; w < busy; ++w)
            most_of_all = __builtin_fmaxf(most_of_all, top[w][own_column]);
        const float scale = exp2_of(m - most_of_all);
        float *to = outs + (wave * 16 + own_column) * ROW;
#pragma unroll
        for (int p = 0; p < PANELS; ++p)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < EACH; i += 4) {
                    const int e = p * EACH + i;
                    *reinterpret_cast<F4 *>(to + p * 16 * EACH + (4 * own_quarter + r) * EACH + i) =
                        F4{o[e][r], o[e + 1][r], o[e + 2][r], o[e + 3][r]} * scale;
                }
    }
    __syncthreads();
    for (int i = thread; i < heads * fours; i += kThreads) {
        const int h = i / fours, at = 4 * (i - h * fours);
        float most_of_all = top[0][h];
        for (int w = 1; w < busy; ++w) most_of_all = __builtin_fmaxf(most_of_all, top[w][h]);
        float whole = 0.f;
        F4 f = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < busy; ++w) {
            whole += sum[w][h] * exp2_of(top[w][h] - most_of_all);
            f += *reinterpret_cast<const F4 *>(outs + (w * 16 + h) * ROW + at);
        }
        const int64_t row = t * a.q_heads + first_head + h;
        if (splits > 1) {
            float *ws = static_cast<float *>(a.workspace);
            const int64_t part = row * splits + piece;
            *reinterpret_cast<F4 *>(ws + n.at_outs + part * a.head_dim + at) = f;
            if (at == 0) {
                ws[2 * part] = most_of_all - UP;
                ws[2 * part + 1] = whole;
            }
        } else {
            const Close c = close_row(n, first_head + h, most_of_all - UP, whole);
            store4<D>(a.out, t * a.out_stride + static_cast<int64_t>(first_head + h) * a.head_dim +
                                 at, f * c.inverse);
            if (a.lse && at == 0) a.lse[row] = c.lse;
        }
    }
}

// A row's chunks, joined in ascending order: sixteen bytes of the output a lane, `wide`
// lanes, chunks dealt to as many groups of lanes as there are.
template <int D>
__global__ void __launch_bounds__(kThreads) join_kernel(const AttendArgs n, const int wide) {
    __shared__ float part[2 * kWaves];
    __shared__ alignas(16) F4 sums[kThreads];
    const sifar_paged_attention_args &a = n.a;
    const int64_t t = blockIdx.y;
    const int head = blockIdx.x, splits = static_cast<int>(n.splits.d);
    const int wave = threadIdx.x / 64, waves = blockDim.x / 64, threads = blockDim.x;
    const Stretch s = stretch(n, t);
    const int chunks = (s.count + s.chunk - 1) / s.chunk;
    const int64_t row = t * a.q_heads + head;
    const float *ml = static_cast<const float *>(a.workspace) + 2 * row * splits;
    const float *outs =
        static_cast<const float *>(a.workspace) + n.at_outs + row * splits * a.head_dim;
    const int lane = threadIdx.x & (wide - 1), group = threadIdx.x / wide;
    const int groups = threads / wide;
    const int at = 4 * (wide * static_cast<int>(blockIdx.z) + lane);
    const bool in = at < a.head_dim;

    // The first chunks' outputs are on their way while the maxima are looked through.
    constexpr int AHEAD = 4;
    F4 x[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
        const int i = group + j * groups;
        x[j] = *reinterpret_cast<const F4 *>(
            outs + static_cast<int64_t>(i < chunks ? i : 0) * a.head_dim + (in ? at : 0));
    }
    float m = kLowest, l = 0.f;
    for (int i = threadIdx.x; i < chunks; i += threads) m = __builtin_fmaxf(m, ml[2 * i]);
    m = wave_reduce(m, [](float x, float y) { return __builtin_fmaxf(x, y); });
    if (waves > 1) {
        if ((threadIdx.x & 63) == 0) part[wave] = m;
        __syncthreads();
        for (int w = 0; w < waves; ++w) m = __builtin_fmaxf(m, part[w]);
    }
    for (int i = threadIdx.x; i < chunks; i += threads) l += ml[2 * i + 1] * exp2_of(ml[2 * i] - m);
    l = wave_reduce(l, Add{});
    if ((threadIdx.x & 63) == 0) part[kWaves + wave] = l;

    F4 f = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
        const int i = group + j * groups;
        if (i < chunks) f += x[j] * exp2_of(ml[2 * i] - m);
    }
#pragma unroll 4
    for (int i = group + AHEAD * groups; i < chunks; i += groups)
        f += *reinterpret_cast<const F4 *>(outs + static_cast<int64_t>(i) * a.head_dim +
                                           (in ? at : 0)) * exp2_of(ml[2 * i] - m);
    sums[threadIdx.x] = f;
    __syncthreads();
    if (group != 0 || !in) return;
    l = part[kWaves];
    for (int w = 1; w < waves; ++w) l += part[kWaves + w];
    for (int g = 1; g < groups; ++g) f += sums[g * wide + lane];
    const Close c = close_row(n, head, m, l);
    store4<D>(a.out, t * a.out_stride + static_cast<int64_t>(head) * a.head_dim + at,
              f * c.inverse);
    if (a.lse && at == 0) a.lse[row] = c.lse;
}

template <int D, int DIM>
void launch_attend(const AttendArgs &n, bool once, dim3 grid, hipStream_t s) {
    if (n.a.head_dim != DIM) attend_kernel<D, DIM, true, false><<<grid, kThreads, 0, s>>>(n);
    else if (once) attend_kernel<D, DIM, false, true><<<grid, kThreads, 0, s>>>(n);
    else attend_kernel<D, DIM, false, false><<<grid, kThreads, 0, s>>>(n);
}

int64_t reach_of(const sifar_paged_attention_args &a) {
    const int64_t slots = static_cast<int64_t>(a.max_pages) * a.page_size;
    return a.max_length < slots ? a.max_length : slots;
}

int64_t most_of(const sifar_paged_attention_args &a) {
    const int64_t reach = reach_of(a);
    return a.window > 0 && a.window < reach ? a.window : reach;
}

template <int D>
hipError_t launch(const sifar_paged_attention_args &a, hipStream_t s) {
    const int64_t splits =
        splits_of(a.dtype, a.tokens, a.q_heads, a.kv_heads, a.head_dim, most_of(a));
    AttendArgs n{};
    n.a = a;
    n.page = make_div(static_cast<uint32_t>(a.page_size));
    n.splits = make_div(static_cast<uint32_t>(splits));
    n.group = a.q_heads / a.kv_heads;
    n.reach = static_cast<int32_t>(reach_of(a));
    n.round = kWaves * tile_of(a.dtype, wide_of(a.head_dim));
    n.unit = __builtin_fabsf(a.scale) > kFar || a.softcap > kFar ? 1.f : kLog2e;
    n.at_outs = outs_at(static_cast<int64_t>(a.tokens) * a.q_heads, splits);
    const dim3 grid(splits, a.kv_heads * tiles_of(a.q_heads, a.kv_heads), a.tokens);
    const int dim = wide_of(a.head_dim);
    // More keys and values than half of the 256 MB cache behind the L2s, read by one
    // workgroup each, go past it: 1 x 131072 (32 heads on 8 of 128, bf16) took 106 us through
    // the caches and 96 past them. Those of 34 MB are read again from there (13.4 and 13.9).
    // Padded heads have no such variant: 64 x 8192 at heads of 96 runs at 4.9 TB/s.
    const bool once = tiles_of(a.q_heads, a.kv_heads) == 1 &&
                      2 * most_of(a) * a.tokens * a.kv_heads * a.head_dim *
                              static_cast<int64_t>(size_of(a.dtype)) >= int64_t{1} << 27;
    if (dim == 64) launch_attend<D, 64>(n, once, grid, s);
    else if (dim == 128) launch_attend<D, 128>(n, once, grid, s);
    else launch_attend<D, 256>(n, once, grid, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    // Few rows, of many chunks each: their outputs in pieces, with many lanes for the chunks.
    if (static_cast<int64_t>(a.tokens) * a.q_heads < 256)
        join_kernel<D><<<dim3(a.q_heads, a.tokens, dim / 32), kThreads, 0, s>>>(n, 8);
    else
        join_kernel<D><<<dim3(a.q_heads, a.tokens), kRowWave, 0, s>>>(n, dim / 4);
    return hipGetLastError();
}

bool good_sizes(int64_t tokens, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                int64_t max_length) {
    return tokens >= 0 && tokens <= SIFAR_ATTENTION_MAX_TOKENS && kv_heads >= 1 &&
           kv_heads <= SIFAR_CACHE_MAX_HEADS && q_heads >= 1 && q_heads <= SIFAR_CACHE_MAX_HEADS &&
           q_heads % kv_heads == 0 && head_dim >= 8 && head_dim <= SIFAR_CACHE_MAX_DIM &&
           head_dim % 8 == 0 && max_length >= 1 && max_length <= SIFAR_ATTENTION_MAX_LENGTH;
}

bool good(const sifar_paged_attention_args &a) {
    if (!good_dtype(a.dtype) ||
        !good_sizes(a.tokens, a.q_heads, a.kv_heads, a.head_dim, a.max_length))
        return false;
    if (a.page_size < 1 || a.page_size > SIFAR_CACHE_MAX_PAGE || a.num_pages < 1 ||
        a.max_pages < 1)
        return false;
    if (a.window < 0 || !__builtin_isfinite(a.scale) || !(a.softcap >= 0.f) ||
        !__builtin_isfinite(a.softcap))
        return false;
    const Paged cache = paged(a.num_pages, a.page_size, a.kv_heads, a.page_stride, a.slot_stride,
                              a.head_stride, a.head_dim);
    const int64_t elements = extent(cache);
    if (elements == 0) return false;
    if (!good_table(a.tokens, a.pages_stride)) return false;
    if (a.tokens == 0) return true;
    if (!a.q || !a.k_cache || !a.v_cache || !a.pages || !a.lengths || !a.out) return false;
    for (const void *p : {a.q, a.k_cache, a.v_cache, static_cast<const void *>(a.out),
                          static_cast<const void *>(a.workspace)})
        if (!aligned16(p)) return false;
    for (const void *p : {static_cast<const void *>(a.pages), static_cast<const void *>(a.lengths),
                          static_cast<const void *>(a.sinks), static_cast<const void *>(a.lse)})
        if (!aligned4(p)) return false;
    const int64_t width = static_cast<int64_t>(a.q_heads) * a.head_dim;
    if (!good_stride(a.q_stride, a.tokens, width) || !good_stride(a.out_stride, a.tokens, width))
        return false;
    const int64_t splits =
        splits_of(a.dtype, a.tokens, a.q_heads, a.kv_heads, a.head_dim, most_of(a));
    const int64_t need = sifar_paged_attention_workspace(a.tokens, a.q_heads, a.kv_heads,
                                                         a.head_dim, a.max_length);
    const int64_t used = used_bytes(static_cast<int64_t>(a.tokens) * a.q_heads, splits, a.head_dim);
    if (splits > 1 && (!a.workspace || a.workspace_bytes < need || need < used)) return false;

    const uint64_t size = size_of(a.dtype), tokens = static_cast<uint64_t>(a.tokens);
    const Rows q = rows_of(a.q, a.dtype, a.tokens, a.q_stride, width);
    const Rows out[] = {rows_of(a.out, a.dtype, a.tokens, a.out_stride, width),
                        span_of(a.lse, a.lse ? 4 * tokens * a.q_heads : 0),
                        span_of(a.workspace, splits > 1 ? static_cast<uint64_t>(need) : 0)};
    const Rows in[] = {span_of(a.k_cache, static_cast<uint64_t>(elements) * size),
                       span_of(a.v_cache, static_cast<uint64_t>(elements) * size),
                       table_of(a.pages, a.tokens, a.pages_stride, a.max_pages),
                       span_of(a.lengths, 4 * tokens),
                       span_of(a.sinks, a.sinks ? 4ull * a.q_heads : 0)};
    for (int o = 0; o < 3; ++o) {
        for (const Rows &i : in)
            if (may_overlap(out[o], i)) return false;
        for (int p = 0; p < o; ++p)
            if (may_overlap(out[o], out[p])) return false;
        if (may_overlap(out[o], q) && !(o == 0 && same_rows(out[o], q))) return false;
    }
    return true;
}

}  // namespace
}  // namespace sifar

extern "C" int64_t sifar_paged_attention_workspace(int32_t tokens, int32_t q_heads,
                                                   int32_t kv_heads, int32_t head_dim,
                                                   int32_t max_length) {
    using namespace sifar;
    if (!good_sizes(tokens, q_heads, kv_heads, head_dim, max_length)) return SIFAR_EINVAL;
    return asked_bytes(tokens, q_heads, kv_heads, head_dim, max_length);
}

extern "C" int sifar_paged_attention(const sifar_paged_attention_args *args, void *stream) {
    using namespace sifar;
    if (!args || !good(*args)) return SIFAR_EINVAL;
    const sifar_paged_attention_args &a = *args;
    if (a.tokens == 0) return SIFAR_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = a.dtype == SIFAR_FP32   ? launch<SIFAR_FP32>(a, s)
                         : a.dtype == SIFAR_BF16 ? launch<SIFAR_BF16>(a, s)
                                                 : launch<SIFAR_FP16>(a, s);
    return e == hipSuccess ? SIFAR_OK : SIFAR_EHIP;
}
