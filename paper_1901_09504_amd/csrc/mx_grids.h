// Grids per block of 32 columns: 4-bit floating-point codes (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) on a power of two
// per block (e8m0: byte b stands for 2^(b - 127), 255 for NaN).  What the passes, the product that does it itself and the cache share.
#pragma once

#include "row_types.h"

namespace ocs {

constexpr int kMxBlock = 32;

struct MxRows {
    const void* X;
    int64_t ldx, M;
    int C, g, s;
    const int32_t* chan_src;
    const int32_t* chan_depth;
    uint8_t* q;                       // two codes a byte, the even column in the low half
    int64_t ldq;
    uint8_t* scale;
    int64_t lds;
};

// Workgroup ids are dealt to the 8 XCDs in turn, each with an L2 of its own.  The id that gives an XCD a run of neighbours instead, which share
// lines of memory (4096 x 4096 bf16 quantized: 63 MB of lines asked of memory and 11.7 us without it, 43 and 10.3 with it).
__device__ __forceinline__ unsigned neighbours_on_an_xcd(unsigned w, unsigned total) {
    const unsigned each = total / 8, more = total % 8, xcd = w % 8;
    return xcd * each + (xcd < more ? xcd : more) + w / 8;
}

// The scale byte of a block whose largest magnitude has these bits: 2^(floor(log2 max) - 2) puts it into [4, 8), the binade of the
// largest code; the exponent field is that logarithm already.  Below 2^-125 the byte ends at 0.  NaN comes above infinity.
__device__ __forceinline__ unsigned mx_scale_byte(unsigned magnitude) {
    const unsigned e = magnitude >> 23;
    return e == 255u ? 255u : (e > 2u ? e - 2u : 0u);
}

// The power of two of a scale byte as the conversions take it: they look at the exponent field alone, 0 for 2^-127 and 255 for NaN.
__device__ __forceinline__ float mx_scale_value(unsigned byte) { return __uint_as_float(byte << 23); }

// Codes of eight values, first in the low bits: the hardware's conversion, nearest, halves to the even code, at most 6.
__device__ __forceinline__ unsigned mx_codes8(const float (&v)[8], float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
    unsigned r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], scale, 3);
#else
    (void)v;
    (void)scale;
    return 0u;
#endif
}

typedef float f32x2 __attribute__((ext_vector_type(2)));

// What eight codes stand for (NaN on scale 255).
__device__ __forceinline__ void mx_values8(unsigned codes, unsigned byte, float (&v)[8]) {
#if defined(__HIP_DEVICE_COMPILE__)
    const float scale = mx_scale_value(byte);
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1),
                c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
    const float all[8] = {a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = all[e];
#else
    (void)codes;
    (void)byte;
    (void)v;
#endif
}

__device__ __forceinline__ unsigned mx_magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// The largest over each four neighbouring lanes.
__device__ __forceinline__ unsigned quad_max(unsigned v) {
    unsigned o = (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);     // lanes 1 0 3 2
    v = o > v ? o : v;
    o = (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);              // lanes 2 3 0 1
    return o > v ? o : v;
}

// 2^-d for a channel's halvings
__device__ __forceinline__ float mx_halvings(int d) { return ldexpf(1.0f, -(d < 0 ? 0 : (d > 255 ? 255 : d))); }

// The channels that expanded columns k0 .. k0 + 7 copy (g = 1) or the columns themselves: what is looked up ahead of the values.
struct MxSources {
    int at[8];
};
typedef int i32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ MxSources mx_sources(const MxRows& p, int k0) {
    const int K = p.C * p.g, Ke = (p.C + p.s) * p.g;
    MxSources s;
    if (p.g == 1 && k0 + 8 <= Ke) {
        const i32x4_a4 a = *reinterpret_cast<const i32x4_a4*>(p.chan_src + k0), b = *reinterpret_cast<const i32x4_a4*>(p.chan_src + k0 + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) s.at[e] = e < 4 ? a[e & 3] : b[e & 3];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int k = k0 + e < Ke ? k0 + e : Ke - 1;
            s.at[e] = k < K ? (p.g == 1 ? k : k / p.g) : p.chan_src[p.g == 1 ? k : k / p.g];
        }
    }
    return s;
}

// Columns k0 .. k0 + 7 of an expanded row, with their halvings; past its end zeros.  The first C * g columns are the row's own: whole
// pieces of it are loaded as they are.  Lanes behind them ask for their sources first, so that those come while the others' pieces do.
template <Elem T, bool SCALED>
__device__ __forceinline__ void mx_expanded8(const MxRows& p, const elem_t<T>* x, int k0, bool there, float (&v)[8]) {
    const int K = p.C * p.g, Ke = (p.C + p.s) * p.g;
    const bool own = there && k0 + 8 <= K, looked = there && !own && k0 < Ke;
    MxSources s;
    u32x4 pieces[8 / kVec<T>];
    if (looked) s = mx_sources(p, k0);
#pragma unroll
    for (int h = 0; h < 8 / kVec<T>; ++h) {
        pieces[h] = u32x4{0u, 0u, 0u, 0u};
        if (own) pieces[h] = load_piece<T>(x + k0 + h * kVec<T>);
    }
    elem_t<T> copies[8];
    if (looked) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int k = k0 + e < Ke ? k0 + e : Ke - 1;
            int src = s.at[e];
            src = src < 0 ? 0 : (src >= p.C ? p.C - 1 : src);
            copies[e] = x[k < K ? k : (p.g == 1 ? src : src * p.g + k % p.g)];
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = piece_elem<T>(pieces[e / kVec<T>], e % kVec<T>);
    if (looked) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k0 + e < Ke ? elem_to_float<T>(copies[e]) : 0.0f;
    }
    if constexpr (SCALED) {
        if (there && p.g == 1 && k0 + 8 <= Ke) {
            const i32x4_a4 a = *reinterpret_cast<const i32x4_a4*>(p.chan_depth + k0), b = *reinterpret_cast<const i32x4_a4*>(p.chan_depth + k0 + 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= mx_halvings(e < 4 ? a[e & 3] : b[e & 3]);
        } else if (there) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (k0 + e < Ke) v[e] *= mx_halvings(p.chan_depth[p.g == 1 ? k0 + e : (k0 + e) / p.g]);
        }
    }
}

}  // namespace ocs
