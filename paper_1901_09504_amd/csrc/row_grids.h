// Rows that are put on grids of their own: what the pass over them and the product that does it itself share.
#pragma once

#include "row_types.h"

namespace ocs {

struct RowGrids {
    const void* X;
    int64_t ldx, M;
    int C, g, s;
    const int32_t* chan_src;
    const int32_t* chan_depth;
    float clip, qmax;
    int8_t* Xq;
    int64_t ldq;
    float* step;
};

// the column that expanded column k copies, and its channel
__device__ __forceinline__ int source_column(const RowGrids& p, int k, int* channel) {
    const int j = p.g == 1 ? k : k / p.g;
    int src = p.chan_src[j];
    src = src < 0 ? 0 : (src >= p.C ? p.C - 1 : src);
    *channel = j;
    return p.g == 1 ? src : src * p.g + (k - j * p.g);
}

// The sources of columns k0 .. k0 + 3, those up to K being their own: four look-ups under way at once, whatever the columns are.
struct FourSources {
    int src[4], channel[4];
};
__device__ __forceinline__ FourSources four_sources(const RowGrids& p, int k0, int K, int Ke) {
    FourSources f;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        f.src[b] = k0 + b;
        f.channel[b] = 0;
    }
    if (p.s == 0 || k0 + 3 < K || k0 >= Ke) return f;
    int looked[4], at[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const int k = k0 + b < Ke ? k0 + b : Ke - 1;
        looked[b] = source_column(p, k, &at[b]);
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        f.src[b] = k0 + b < K ? k0 + b : looked[b];
        f.channel[b] = at[b];
    }
    return f;
}

__device__ __forceinline__ float depth_factor(const RowGrids& p, int channel) {
    int d = p.chan_depth[channel];
    d = d < 0 ? 0 : (d > 255 ? 255 : d);
    return ldexpf(1.0f, -d);
}

// magnitudes as whole numbers: they order like them, and NaN comes above infinity
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

}  // namespace ocs
