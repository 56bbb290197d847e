// Element types of the calls with a grid per row and of token scoring: 16-byte pieces of fp32, bf16 or fp16 rows at any
// alignment of the element, as fp32 numbers and back.
#pragma once

#include "ocs_internal.h"

namespace ocs {

enum class Elem { f32 = 0, bf16 = 1, f16 = 2 };   // OCS_F32, OCS_BF16, OCS_F16

template <Elem T>
struct ElemOf;
template <>
struct ElemOf<Elem::f32> {
    using type = float;
};
template <>
struct ElemOf<Elem::bf16> {
    using type = unsigned short;
};
template <>
struct ElemOf<Elem::f16> {
    using type = _Float16;
};
template <Elem T>
using elem_t = typename ElemOf<T>::type;
template <Elem T>
constexpr int kVec = 16 / (int)sizeof(elem_t<T>);   // elements of a 16-byte piece

// Global memory serves 16 bytes at any address (the mode that the ROCm runtime sets for gfx9); the types only tell the compiler.
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned u32x2_a4 __attribute__((ext_vector_type(2), aligned(4)));
typedef unsigned u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));

template <Elem T>
__device__ __forceinline__ u32x4 load_piece(const elem_t<T>* p) {
    if constexpr (T == Elem::f32) return *reinterpret_cast<const u32x4_a4*>(p);
    else return *reinterpret_cast<const u32x4_a2*>(p);
}

template <Elem T>
__device__ __forceinline__ float elem_to_float(elem_t<T> v) {
    if constexpr (T == Elem::bf16) return __uint_as_float((unsigned)v << 16);
    else return (float)v;
}

// element e of a piece
template <Elem T>
__device__ __forceinline__ float piece_elem(u32x4 p, int e) {
    if constexpr (T == Elem::f32) {
        return __uint_as_float(p[e]);
    } else if constexpr (T == Elem::bf16) {
        return __uint_as_float((e & 1) ? p[e / 2] & 0xFFFF0000u : p[e / 2] << 16);
    } else {
        return (float)__builtin_bit_cast(_Float16, (unsigned short)((e & 1) ? p[e / 2] >> 16 : p[e / 2] & 0xFFFFu));
    }
}

// a 16-byte piece of which the first n elements are in the row (0 < n < kVec): the rest reads as zero
template <Elem T>
__device__ __forceinline__ u32x4 load_partial(const elem_t<T>* p, int n) {
    u32x4 r = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) {
        if (e >= n) break;
        if constexpr (T == Elem::f32) r[e] = __float_as_uint(p[e]);
        else r[e / 2] |= (unsigned)__builtin_bit_cast(unsigned short, p[e]) << (16 * (e & 1));
    }
    return r;
}

// fp32 to the output type, rounded once, half to even
template <Elem T>
__device__ __forceinline__ elem_t<T> float_to_elem(float v) {
    if constexpr (T == Elem::bf16) return __builtin_bit_cast(unsigned short, (__bf16)v);
    else return (elem_t<T>)v;
}

// kVec elements to any address of the element's alignment
template <Elem T>
__device__ __forceinline__ void store_piece(elem_t<T>* p, const elem_t<T> (&v)[kVec<T>]) {
    u32x4 r;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        if constexpr (T == Elem::f32)
            r[d] = __float_as_uint(v[d]);
        else
            r[d] = (unsigned)__builtin_bit_cast(unsigned short, v[2 * d]) | (unsigned)__builtin_bit_cast(unsigned short, v[2 * d + 1]) << 16;
    }
    if constexpr (T == Elem::f32) *reinterpret_cast<u32x4_a4*>(p) = r;
    else *reinterpret_cast<u32x4_a2*>(p) = r;
}

}  // namespace ocs
