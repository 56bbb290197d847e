// What the products of row-wise code tensors share: pieces of codes from memory into LDS, which tile a workgroup takes, how the outputs
// are dealt over a tile's rows.
#pragma once

#include <atomic>

#include "row_types.h"

namespace ocs {

// What a row "holds" past its pitch, where that ends inside the last step.
static __device__ __align__(16) int8_t rows_zero_chunk[16] = {};

// 1 KB of codes, 16 bytes per lane, from each lane's address to LDS at lds_addr + 16 * lane.  Issued by hand because the compiler
// waits for all of its own before every read of LDS; the waits are wait_requests below.
__device__ __forceinline__ void request_1k(const int8_t* from, unsigned lds_addr) {
#if defined(__HIP_DEVICE_COMPILE__)
    const unsigned m0 = __builtin_amdgcn_readfirstlane(lds_addr);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(m0) : "memory");
#else
    (void)from;
    (void)lds_addr;
#endif
}

// The same from a wave-uniform base and each lane's offset (no vector arithmetic from step to step).
__device__ __forceinline__ void request_1k(const int8_t* base, unsigned offset, unsigned lds_addr) {
#if defined(__HIP_DEVICE_COMPILE__)
    const unsigned m0 = __builtin_amdgcn_readfirstlane(lds_addr);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(m0) : "memory");
#else
    (void)base;
    (void)offset;
    (void)lds_addr;
#endif
}

// 64 words, one per lane.
__device__ __forceinline__ void request_256(const float* from, unsigned lds_addr) {
#if defined(__HIP_DEVICE_COMPILE__)
    const unsigned m0 = __builtin_amdgcn_readfirstlane(lds_addr);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(from), "s"(m0) : "memory");
#else
    (void)from;
    (void)lds_addr;
#endif
}

// until at most N of this wave's requests are under way
template <int N>
__device__ __forceinline__ void wait_requests() {
    static_assert(N >= 0 && N < 64, "a 6-bit counter");
    __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ unsigned lds_address(const int8_t* p) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __attribute__((address_space(3))) const int8_t* lptr_t;
    return (unsigned)(uintptr_t)(lptr_t)p;
#else
    (void)p;
    return 0;
#endif
}

// fp32: outputs of a token lie 4 to a lane.  Two-byte outputs: the rows of two neighbouring weight tiles are dealt so that a lane
// has 8 in a row, 16 bytes either way.  Row R of the tiles' image holds output column_of(R).
template <Elem OUT>
__device__ __forceinline__ int column_of(int R) {
    if constexpr (OUT == Elem::f32) return R;
    else return (R & ~31) + ((R & 15) >> 2) * 8 + ((R >> 4) & 1) * 4 + (R & 3);
}

typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

// p[at .. at + 3] of an array of n floats (what lies past it is never used)
__device__ __forceinline__ f32x4 four_of(const float* p, int at, int n) {
    if (at + 4 <= n) return *reinterpret_cast<const f32x4_a4*>(p + at);
    f32x4 r = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (at + e < n) r[e] = p[at + e];
    return r;
}

// Workgroup ids are dealt to the 8 XCDs in turn, each with an L2 of its own.  An XCD gets a run of tiles, and the run goes down
// kTileRows rows of tiles before it goes to the next column: what runs at one time on an XCD is a block of tiles, whose panels of X and
// W the L2 holds for all of them.
constexpr int kTileRows = 8;
__device__ __forceinline__ void tile_of(unsigned w, int tiles_m, int tiles_n, int* bm, int* bn) {
    const unsigned total = (unsigned)tiles_m * (unsigned)tiles_n, each = total / 8, more = total % 8, xcd = w % 8;
    const unsigned id = xcd * each + (xcd < more ? xcd : more) + w / 8;
    const unsigned band = (unsigned)kTileRows * (unsigned)tiles_n, b = id / band, in = id - b * band;
    const unsigned first = b * kTileRows, rows = (unsigned)tiles_m - first < kTileRows ? (unsigned)tiles_m - first : kTileRows;
    *bm = (int)(first + in % rows);
    *bn = (int)(in / rows);
}

// Pitches from here on have offsets inside a tile that do not fit 32 bits.
constexpr int64_t kWidePitch = (int64_t)1 << 24;

constexpr int kMostLds = 160 * 1024;   // of a compute unit

// Lets a kernel have `bytes` of LDS by its launch, once per device.
static hipError_t allow_lds(const void* kernel, int bytes, std::atomic<bool>* allowed) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
    if (allowed[dev].load(std::memory_order_acquire)) return hipSuccess;
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) allowed[dev].store(true, std::memory_order_release);
    return e;
}

}  // namespace ocs
