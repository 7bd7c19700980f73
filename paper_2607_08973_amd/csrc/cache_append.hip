// Keys and values of new tokens into a paged cache, rotated by their positions on the
// way, and the queries rotated beside them: sifar_cache_append. gfx950 (MI355X) only.
//
// A workgroup holds one token. Its angles, one for each pair of a head's rotated
// elements, are the same for all heads: as many lanes as there are pairs compute
// cosine and sine once and leave them in LDS, while every lane's own elements are on
// their way. Each input is read once and each output written once. Bound: HBM bytes for
// many tokens; for a few the launch and two dependent round trips (the position, then
// its page). Measured: 8192 tokens of 32 + 2 x 8 heads of 128, bf16, 39.7 us a call, 5.1
// TB/s, the rate of a copy; in a graph 1 token 3.0 us, 77 tokens (12 + 2 x 4 heads of 96) 3.2.
//
// Angles: position times frequency is formed in 64 bits and reduced to a quadrant there,
// so that a position of a million is as exact as one of ten; what remains of the angle,
// within pi/4, goes through fp32 polynomials.
#include <hip/hip_runtime.h>

#include "paged.h"
#include "rows.h"
#include "sifar_kernels.h"

namespace sifar {
namespace {

constexpr int kMaxThreads = 1024;
constexpr int kMaxPairs = SIFAR_CACHE_MAX_DIM / 2;

struct AppendArgs {
    sifar_cache_append_args a;
    DivU32 page;   // by page_size
    DivU32 head;   // by the items of a rotated head
    DivU32 value;  // by the items of a head of values
    int32_t rotated, items;  // items of q and k, of all three
};

// VEC adjacent elements, as they are stored.
template <int D, int VEC>
struct Part {
    Stored<D> e[VEC];
};

template <int D, int VEC>
__device__ __forceinline__ Part<D, VEC> load_part(const void *row, int64_t at) {
    constexpr int align = sizeof(Part<D, VEC>) < 16 ? sizeof(Part<D, VEC>) : 16;
    Part<D, VEC> p;
    __builtin_memcpy(&p, __builtin_assume_aligned(static_cast<const Stored<D> *>(row) + at, align),
                     sizeof(p));
    return p;
}

template <int D, int VEC>
__device__ __forceinline__ void store_part(void *row, int64_t at, const Part<D, VEC> &p) {
    constexpr int align = sizeof(Part<D, VEC>) < 16 ? sizeof(Part<D, VEC>) : 16;
    __builtin_memcpy(__builtin_assume_aligned(static_cast<Stored<D> *>(row) + at, align), &p,
                     sizeof(p));
}

template <int D>
__device__ __forceinline__ Stored<D> narrow(float f) {
    if constexpr (D == SIFAR_FP32) return __float_as_uint(f);
    else return static_cast<uint16_t>(pack16<D>(f, f));
}

// Cosine and sine of an angle in 64 bits: the nearest multiple of pi/2 and what is left,
// whose Taylor series to x^9 and x^10 are off by less than 2e-9 for |x| <= pi/4.
__device__ __forceinline__ void turn(double angle, float *cosine, float *sine) {
    const double t = angle * 0x1.45f306dc9c883p-1;  // 2 / pi
    const double q = __builtin_rint(t);
    const float x = static_cast<float>(t - q) * 0x1.921fb6p+0f;  // pi / 2
    const float y = x * x;
    float s = 0x1.71de3ap-19f;  // 1 / 9!
    s = __builtin_fmaf(s, y, -0x1.a01a02p-13f);
    s = __builtin_fmaf(s, y, 0x1.111112p-7f);
    s = __builtin_fmaf(s, y, -0x1.555556p-3f);
    s = __builtin_fmaf(s * y, x, x);
    float c = -0x1.27e4fcp-22f;  // -1 / 10!
    c = __builtin_fmaf(c, y, 0x1.a01a02p-16f);
    c = __builtin_fmaf(c, y, -0x1.6c16c2p-10f);
    c = __builtin_fmaf(c, y, 0x1.555556p-5f);
    c = __builtin_fmaf(c, y, -0.5f);
    c = __builtin_fmaf(c, y, 1.f);
    const int k = static_cast<int>(q - 4.0 * __builtin_floor(0.25 * q));  // 0..3
    const float a = k & 1 ? s : c, b = k & 1 ? c : s;
    *cosine = k == 1 || k == 2 ? -a : a;
    *sine = k >= 2 ? -b : b;
}

// D: element type. VEC: adjacent elements of an item, which holds VEC pairs (their two
// halves of the rotated part lie rotary_dim / 2 apart) or VEC elements that are copied.
// ADJACENT: pairs of adjacent elements, VEC / 2 of them an item.
template <int D, int VEC, bool ADJACENT>
__global__ void __launch_bounds__(kMaxThreads) append_kernel(const AppendArgs n) {
    __shared__ float cosine[kMaxPairs], sine[kMaxPairs];
    const sifar_cache_append_args &a = n.a;
    const int64_t t = blockIdx.x;
    const int position = a.positions[t];
    if (position < 0) return;  // the same for the workgroup
    const int pairs = a.rotary_dim / 2;
    // of a head: items with pairs, then items that are copied
    const int turned = ADJACENT ? 0 : pairs / VEC;

    struct Item {
        const void *from;  // the head's first element
        int64_t row;       // of it, in elements
        int head, at;      // of q, k or v: 0.. in that order; first element, or first pair
        bool pair, value;
    };
    const auto item_of = [&](int i) {
        Item m;
        m.value = i >= n.rotated;
        const int j = m.value ? i - n.rotated : i;
        const DivU32 &div = m.value ? n.value : n.head;
        const int head = static_cast<int>(div_u32(static_cast<uint32_t>(j), div));
        const int k = j - head * static_cast<int>(div.d);
        m.pair = !m.value && (ADJACENT ? k * VEC < 2 * pairs : k < turned);
        m.at = VEC * k + (!ADJACENT && !m.value && k >= turned ? pairs : 0);
        m.head = m.value ? a.q_heads + a.kv_heads + head : head;
        const bool q = !m.value && head < a.q_heads;
        m.from = m.value ? a.v : q ? a.q : a.k;
        m.row = t * (m.value ? a.v_stride : q ? a.q_stride : a.k_stride) +
                static_cast<int64_t>(m.value || q ? head : head - a.q_heads) * a.head_dim;
        return m;
    };
    int i = threadIdx.x;
    Item m = item_of(i < n.items ? i : 0);
    Part<D, VEC> x = load_part<D, VEC>(m.from, m.row + m.at), y;
    if (!ADJACENT) y = load_part<D, VEC>(m.from, m.row + m.at + (m.pair ? pairs : 0));

    const int sequence = a.sequence ? a.sequence[t] : static_cast<int>(t);
    const uint32_t nth = div_u32(static_cast<uint32_t>(position), n.page);
    int page = -1;
    if (static_cast<uint32_t>(sequence) < static_cast<uint32_t>(a.sequences) &&
        nth < static_cast<uint32_t>(a.max_pages))
        page = a.pages[sequence * a.pages_stride + nth];
    const bool there = static_cast<uint32_t>(page) < static_cast<uint32_t>(a.num_pages);
    const int64_t slot = page * a.page_stride +
                         static_cast<int64_t>(position - nth * n.page.d) * a.slot_stride;

    for (int p = threadIdx.x; p < pairs; p += blockDim.x) {
        float c, s;
        turn(static_cast<double>(position) * static_cast<double>(a.inv_freq[p]), &c, &s);
        cosine[p] = a.rotary_scale * c;
        sine[p] = a.rotary_scale * s;
    }
    __syncthreads();

    while (i < n.items) {
        Part<D, VEC> u = x, v = y;
        if (m.pair) {
            if constexpr (ADJACENT) {
#pragma unroll
                for (int k = 0; k < VEC; k += 2) {
                    const int p = (m.at + k) / 2;
                    if (p >= pairs) continue;  // behind the rotated part
                    const float f = widen<D>(x.e[k]), g = widen<D>(x.e[k + 1]);
                    u.e[k] = narrow<D>(__builtin_fmaf(f, cosine[p], -(g * sine[p])));
                    u.e[k + 1] = narrow<D>(__builtin_fmaf(f, sine[p], g * cosine[p]));
                }
            } else {
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    const float f = widen<D>(x.e[k]), g = widen<D>(y.e[k]);
                    const float c = cosine[m.at + k], s = sine[m.at + k];
                    u.e[k] = narrow<D>(__builtin_fmaf(f, c, -(g * s)));
                    v.e[k] = narrow<D>(__builtin_fmaf(f, s, g * c));
                }
            }
        }
        const bool q = m.head < a.q_heads;
        const int head = m.value ? m.head - a.q_heads - a.kv_heads
                         : q     ? m.head
                                 : m.head - a.q_heads;
        void *to = m.value ? a.v_cache : q ? a.q_out : a.k_cache;
        const int64_t row = q ? t * a.q_out_stride + static_cast<int64_t>(head) * a.head_dim
                              : slot + head * a.head_stride;
        if (q || there) {
            store_part<D, VEC>(to, row + m.at, u);
            if (!ADJACENT && m.pair) store_part<D, VEC>(to, row + m.at + pairs, v);
        }
        i += blockDim.x;
        if (i >= n.items) break;
        m = item_of(i);
        x = load_part<D, VEC>(m.from, m.row + m.at);
        if (!ADJACENT) y = load_part<D, VEC>(m.from, m.row + m.at + (m.pair ? pairs : 0));
    }
}

template <int D>
hipError_t launch_append(const sifar_cache_append_args &a, hipStream_t s) {
    const int pairs = a.rotary_dim / 2;
    // Both halves of a head's pairs, and what is copied behind them, in vectors of 16
    // bytes (of 16 bits); where the halves are not whole vectors, in smaller ones.
    const int vec = a.interleaved || pairs % 8 == 0 ? 8 : pairs % 4 == 0 ? 4 : 1;
    AppendArgs n{};
    n.a = a;
    const int head = a.interleaved ? a.head_dim / vec
                                   : (a.head_dim - a.rotary_dim) / vec + pairs / vec;
    n.page = make_div(static_cast<uint32_t>(a.page_size));
    n.head = make_div(static_cast<uint32_t>(head));
    n.value = make_div(static_cast<uint32_t>(a.head_dim / vec));
    n.rotated = (a.q_heads + a.kv_heads) * head;
    n.items = n.rotated + a.kv_heads * (a.head_dim / vec);
    const int waves = (n.items + kRowWave - 1) / kRowWave;
    const dim3 grid(a.tokens), block((waves < 16 ? waves : 16) * kRowWave);
    if (a.interleaved) append_kernel<D, 8, true><<<grid, block, 0, s>>>(n);
    else if (vec == 8) append_kernel<D, 8, false><<<grid, block, 0, s>>>(n);
    else if (vec == 4) append_kernel<D, 4, false><<<grid, block, 0, s>>>(n);
    else append_kernel<D, 1, false><<<grid, block, 0, s>>>(n);
    return hipGetLastError();
}

bool good(const sifar_cache_append_args &a) {
    if (!good_dtype(a.dtype) || a.tokens < 0 || a.tokens > SIFAR_ROWS_MAX_TOKENS) return false;
    if (a.kv_heads < 1 || a.kv_heads > SIFAR_CACHE_MAX_HEADS || a.q_heads < 0 ||
        a.q_heads > SIFAR_CACHE_MAX_HEADS)
        return false;
    if (a.head_dim < 8 || a.head_dim > SIFAR_CACHE_MAX_DIM || a.head_dim % 8) return false;
    if (a.rotary_dim < 0 || a.rotary_dim > a.head_dim || a.rotary_dim % 2) return false;
    if (a.interleaved != 0 && a.interleaved != 1) return false;
    if (a.page_size < 1 || a.page_size > SIFAR_CACHE_MAX_PAGE || a.num_pages < 1 ||
        a.max_pages < 1 || a.sequences < 1)
        return false;
    const Paged cache = paged(a.num_pages, a.page_size, a.kv_heads, a.page_stride, a.slot_stride,
                              a.head_stride, a.head_dim);
    const int64_t elements = extent(cache);
    if (elements == 0) return false;
    if (!good_table(a.sequences, a.pages_stride)) return false;
    if (a.tokens == 0) return true;
    if (!a.sequence && a.tokens > a.sequences) return false;
    if (!a.k || !a.v || !a.positions || !a.pages || !a.k_cache || !a.v_cache) return false;
    if ((a.q_heads != 0) != (a.q != nullptr) || (a.q_heads != 0) != (a.q_out != nullptr))
        return false;
    if ((a.rotary_dim != 0) != (a.inv_freq != nullptr)) return false;
    for (const void *p :
         {a.q, static_cast<const void *>(a.q_out), a.k, a.v, static_cast<const void *>(a.k_cache),
          static_cast<const void *>(a.v_cache)})
        if (!aligned16(p)) return false;
    for (const void *p :
         {static_cast<const void *>(a.positions), static_cast<const void *>(a.sequence),
          static_cast<const void *>(a.pages), static_cast<const void *>(a.inv_freq)})
        if (!aligned4(p)) return false;
    const int64_t q_row = static_cast<int64_t>(a.q_heads) * a.head_dim;
    const int64_t k_row = static_cast<int64_t>(a.kv_heads) * a.head_dim;
    if (!good_stride(a.k_stride, a.tokens, k_row) || !good_stride(a.v_stride, a.tokens, k_row))
        return false;
    if (a.q && (!good_stride(a.q_stride, a.tokens, q_row) ||
                !good_stride(a.q_out_stride, a.tokens, q_row)))
        return false;

    // Any workgroup's outputs, against what any other reads or writes.
    const uint64_t size = size_of(a.dtype);
    const Rows q = rows_of(a.q, a.dtype, a.tokens, a.q_stride, q_row);
    const Rows in[] = {rows_of(a.k, a.dtype, a.tokens, a.k_stride, k_row),
                       rows_of(a.v, a.dtype, a.tokens, a.v_stride, k_row),
                       span_of(a.positions, 4ull * a.tokens),
                       span_of(a.sequence, a.sequence ? 4ull * a.tokens : 0),
                       table_of(a.pages, a.sequences, a.pages_stride, a.max_pages),
                       span_of(a.inv_freq, 2ull * a.rotary_dim)};
    const Rows q_out = rows_of(a.q_out, a.dtype, a.tokens, a.q_out_stride, q_row);
    const Rows caches[] = {span_of(a.k_cache, static_cast<uint64_t>(elements) * size),
                           span_of(a.v_cache, static_cast<uint64_t>(elements) * size)};
    const int64_t apart = static_cast<int64_t>(reinterpret_cast<uintptr_t>(a.v_cache) -
                                               reinterpret_cast<uintptr_t>(a.k_cache));
    if (apart % 16 || shares(cache, apart / static_cast<int64_t>(size))) return false;
    if (may_overlap(q_out, q) && !same_rows(q_out, q)) return false;
    for (const Rows &i : in)
        if (may_overlap(q_out, i) || may_overlap(caches[0], i) || may_overlap(caches[1], i))
            return false;
    for (const Rows &c : caches)
        if (may_overlap(c, q) || may_overlap(c, q_out)) return false;
    return true;
}

}  // namespace
}  // namespace sifar

extern "C" int sifar_cache_append(const sifar_cache_append_args *args, void *stream) {
    using namespace sifar;
    if (!args || !good(*args)) return SIFAR_EINVAL;
    const sifar_cache_append_args &a = *args;
    if (a.tokens == 0) return SIFAR_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = a.dtype == SIFAR_FP32   ? launch_append<SIFAR_FP32>(a, s)
                         : a.dtype == SIFAR_BF16 ? launch_append<SIFAR_BF16>(a, s)
                                                 : launch_append<SIFAR_FP16>(a, s);
    return e == hipSuccess ? SIFAR_OK : SIFAR_EHIP;
}
