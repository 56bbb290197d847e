// A quantized key/value cache in pages: what writing, reading and attention share.
//
// Page x of the pool holds P positions of H heads: codes [H, P, D] and their scales, fp32 steps [H, P] (8 bits) or bytes [H, P, D / 32]
// (4 bits).  Position j of sequence b is row j % P of page table[b][j / P].
#pragma once

#include "mx_grids.h"

namespace ocs {

enum class CacheFormat { int8 = 0, mx4 = 1 };   // OCS_CACHE_INT8, OCS_CACHE_MX4

constexpr int kMostPositions = 0x7FFF0000;      // attention's: its next blocks of positions are numbers of 32 bits, too
constexpr int kMostDepth = 126;                 // 2^126 and 2^-126 are normal numbers

struct Cache {
    const int32_t* table;
    int64_t cols, ldt;
    void* keys;
    void* kscales;
    void* values;
    void* vscales;
    int64_t pages;
    int P, H, D;
    const int32_t* kdepth;                      // halvings [H, D] of a channel before its grid, or NULL
    const int32_t* vdepth;
};

// Sequences: tokens cu[b] .. cu[b + 1] - 1 are positions starts[b], starts[b] + 1, ...
struct Sequences {
    int T, B;
    const int32_t* cu;
    const int32_t* starts;
};

__device__ __forceinline__ int clamp_int(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

// How many i < n have key(i) <= t, key ascending: 64 candidates at a time by the whole wave.
template <typename F>
__device__ __forceinline__ int wave_count(int n, F at_most) {
    const int lane = (int)threadIdx.x & 63;
    int lo = 0, left = n;                                       // the answer lies in lo .. lo + left
    while (left > 0) {
        const int step = (left + 63) / 64, i = lo + (lane + 1) * step - 1;      // last of each of 64 runs
        const int runs = __popcll(__ballot(lane * (int64_t)step < left && (i < lo + left ? at_most(i) : at_most(lo + left - 1))));
        // whole runs that are below the answer; the rest of the search is the next run without its last
        if ((int64_t)runs * step >= left) return lo + left;
        lo += runs * step;
        const int run = left - runs * step < step ? left - runs * step : step;
        left = run - 1;
    }
    return lo;
}

// The sequence of token t (the same in the whole wave), or -1 behind the last, and the token's position in it.  Up to 64 sequences are looked
// at once.
__device__ __forceinline__ int sequence_of(const Sequences& q, int t, int64_t* position) {
    int b, first, start;
    if (q.B <= 64) {
        const int lane = (int)threadIdx.x & 63, i = lane < q.B ? lane : q.B - 1;
        const int from = q.cu[i], to = q.cu[i + 1], at = q.starts[i];
        const uint64_t which = __ballot(lane < q.B && from <= t && t < to);
        if (which == 0) return -1;
        b = __builtin_ctzll(which);
        first = __builtin_amdgcn_readlane(from, b);
        start = __builtin_amdgcn_readlane(at, b);
    } else {
        if (q.T == q.B && q.cu[t] == t && q.cu[t + 1] == t + 1) b = t;          // a token each
        else b = wave_count(q.B, [&](int i) { return q.cu[i + 1] <= t; });
        if (b >= q.B) return -1;
        first = q.cu[b];
        start = q.starts[b];
        if (first > t) return -1;
    }
    *position = (int64_t)start + ((int64_t)t - first);
    return b;
}

// The row of position `pos` of sequence b in the pool, counted in [pages, H, P] for head 0, or -1 where there is none.
__device__ __forceinline__ int64_t cache_row(const Cache& c, int b, int64_t pos) {
    if (pos < 0 || pos >= c.cols * c.P) return -1;
    const int64_t col = pos / c.P, page = c.table[b * c.ldt + col];
    if (page < 0 || page >= c.pages) return -1;
    return page * c.H * c.P + (pos - col * c.P);
}

__device__ __forceinline__ float cache_halvings(int d) { return ldexpf(1.0f, -clamp_int(d, 0, kMostDepth)); }
__device__ __forceinline__ float cache_doublings(int d) { return ldexpf(1.0f, clamp_int(d, 0, kMostDepth)); }

}  // namespace ocs
