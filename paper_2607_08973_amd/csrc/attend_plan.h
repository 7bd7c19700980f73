// How sifar_paged_attention shares sequences among workgroups, and what its workspace
// holds. Plain C++ (host; the constants also on the device).
#pragma once

#include <stdint.h>

#include "sifar.h"

namespace sifar {

constexpr int kWaves = 4;
constexpr int kMinChunk = 128;   // positions of a shared sequence's chunk, at least
constexpr int kMaxChunk = 1536;  // and at most
constexpr int kCus = 256;
constexpr int64_t kSmall = 262144;  // bytes of a workgroup's keys and values

// Positions of a tile.
constexpr int tile_of(int dtype, int dim) { return dtype == SIFAR_FP32 || dim > 128 ? 16 : 32; }

// Workgroups that a CU holds at once, as the registers allow.
constexpr int held_by_a_cu(int dtype, int dim, bool padded) {
    return dim == 64    ? (dtype == SIFAR_FP32 && !padded ? 5 : 4)
           : dim == 128 ? 3
                        : (dtype == SIFAR_FP32 ? 1 : 2);
}

constexpr int kMostHeld = 5;

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int64_t tiles_of(int64_t q_heads, int64_t kv_heads) {
    return ceil_div(q_heads / kv_heads, 16);
}

inline int wide_of(int64_t head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

// The most chunks that a sequence is cut into. At least so many that none is above
// kMaxChunk; and then as many as full rounds of the workgroups that the GPU holds at once
// have room for, as long as none is below kMinChunk. A round more is taken where it leaves
// a tenth less of the places empty: 64 x 4096 (64 heads on 8 of 128, bf16) takes 190 us in 3
// chunks (two rounds), 204 in 4 (2.7 rounds). Two rounds are taken where the workgroups of one
// have so little to read that they all start and end together: 16 x 2000 (16 heads of 64) in
// bf16 34.2 us in one, 33.2 in two. (In fp32, where five workgroups a CU make one round of 5
// chunks, it is the other way about: 46.9 and 52.0.)
//
// All of it goes by the most that a length may be: where lengths are far below that, a
// sequence is in smaller chunks than its own length would make, down to kMinChunk, and most
// workgroups read a length and leave. 64 x 1000 (64 heads on 8 of 128, bf16) takes 60 us under
// a max_length of 1024, 69 under 32768, 76 under 131072; 8 x 1000 13, 16 and 30.
inline int64_t splits_of(int dtype, int64_t tokens, int64_t q_heads, int64_t kv_heads,
                         int64_t head_dim, int64_t reach) {
    const int dim = wide_of(head_dim);
    const int64_t held = kCus * held_by_a_cu(dtype, dim, head_dim != dim);
    const int64_t groups = tokens * kv_heads * tiles_of(q_heads, kv_heads);
    // The smallest chunks only where twice as long ones would not give every CU a workgroup:
    // 1 x 2048 takes 9.9 and 10.9 us with 128 and 256, 8 x 4096 33.1 and 32.0 (32 heads on 8).
    const int64_t least =
        groups * ceil_div(reach, 2 * kMinChunk) < kCus ? kMinChunk : 2 * kMinChunk;
    const int64_t fine = ceil_div(reach, least), coarse = ceil_div(reach, kMaxChunk);
    const int64_t round = kWaves * tile_of(dtype, dim);
    int64_t rounds = ceil_div(groups * coarse, held);
    const int64_t bytes = 2 * head_dim * (dtype == SIFAR_FP32 ? 4 : 2);  // of a position
    if (rounds == 1 && groups * reach * bytes < held * kSmall) rounds = 2;
    int64_t best = coarse;
    double best_used = 0.0;
    for (int64_t r = rounds; r < rounds + 2; ++r) {
        int64_t splits = r * held / groups;
        splits = splits > fine ? fine : splits;
        const int64_t chunk = ceil_div(ceil_div(reach, splits), round) * round;
        const int64_t pieces = ceil_div(reach, chunk);
        const double used = static_cast<double>(groups * reach) /
                            static_cast<double>(ceil_div(groups * pieces, held) * held * chunk);
        if (used > 1.1 * best_used) {
            best_used = used;
            best = splits;
        }
    }
    return best;
}

// Positions of a chunk, of a sequence whose even share is `share`; `round` is a power of two
// that kMaxChunk is a multiple of.
constexpr int chunk_of(int share, int round) {
    const int chunk = (share + round - 1) & -round;
    return chunk < kMinChunk ? kMinChunk : chunk;
}

// The workspace: each row's chunks' maxima and sums, then, 16-byte aligned, their outputs.
inline int64_t outs_at(int64_t rows, int64_t splits) { return (2 * rows * splits + 3) / 4 * 4; }

// Bytes that a call uses, and those that it asks for.
inline int64_t used_bytes(int64_t rows, int64_t splits, int64_t head_dim) {
    return splits == 1 ? 0 : 4 * (outs_at(rows, splits) + rows * splits * head_dim);
}

inline int64_t asked_bytes(int64_t tokens, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                           int64_t max_length) {
    if (max_length <= kMinChunk || tokens == 0) return 0;
    // Chunks of all sequences: no more than the smallest make, nor than the largest make and
    // three rounds of the most workgroups that are ever held. Each grows with tokens and
    // max_length.
    const int64_t groups = static_cast<int64_t>(tokens) * kv_heads * tiles_of(q_heads, kv_heads);
    const int64_t fine = groups * ceil_div(max_length, kMinChunk);
    const int64_t full = groups * ceil_div(max_length, kMaxChunk) + 3 * kCus * kMostHeld;
    const int64_t chunks = fine < full ? fine : full;
    // a chunk has a row for each query head of its tile: its maximum, its sum, its output
    const int64_t rows = q_heads / kv_heads < 16 ? q_heads / kv_heads : 16;
    return (chunks * rows * (head_dim + 2) + 4) * 4;
}

}  // namespace sifar
