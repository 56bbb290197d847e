// Rows onto grids per block of 32 columns, and back to numbers.
//
// For expanded column k of row m: x' = X[m, source(k)] * 2^-depth; over a block a = max|x'|, e = floor(log2 a) - 2 (at least -127),
// code = nearest e2m1 number to x' * 2^-e.  Four lanes share a block, 8 columns each: the block's maximum is two exchanges between
// neighbours, loads and stores are whole 16- and 4-byte pieces of consecutive lanes, and nothing waits for a row: bound by HBM for many
// rows (4096 x 4096 bf16 with 82 splits 10.3 us, 4.2 TB/s; back to bf16 8.2, 5.3), by one launch for few (64 x 256 3.2).
#include "mx_grids.h"

namespace ocs {

// `blocks` blocks a row, the padding of codes and scales among them.
template <Elem T, bool SCALED>
__global__ __launch_bounds__(256) void mx_quantize_kernel(MxRows p, unsigned blocks, unsigned magic) {
    const unsigned at = (neighbours_on_an_xcd(blockIdx.x, gridDim.x) * 256 + threadIdx.x) >> 2;      // (kMostLanes fits 32 bits)
    const int part = (int)(threadIdx.x & 3);
    unsigned r = __umulhi(at, magic);                               // at / blocks or one more: magic is 2^32 / blocks and one more, at below 2^30
    int block = (int)(at - r * blocks);
    if (block < 0) {
        r -= 1;
        block += (int)blocks;
    }
    const int64_t row = r, k0 = (int64_t)block * kMxBlock + part * 8;
    if (row >= p.M) return;                                         // whole groups of four
    float v[8];
    mx_expanded8<T, SCALED>(p, static_cast<const elem_t<T>*>(p.X) + row * p.ldx, (int)k0, k0 < (int64_t)(p.C + p.s) * p.g, v);
    unsigned big = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) big = mx_magnitude(v[e]) > big ? mx_magnitude(v[e]) : big;
    const unsigned byte = mx_scale_byte(quad_max(big));
    const unsigned codes = byte == 255u ? 0u : mx_codes8(v, mx_scale_value(byte));
    if ((int64_t)block * 16 < p.ldq) *reinterpret_cast<unsigned*>(p.q + row * p.ldq + (int64_t)block * 16 + part * 4) = codes;
    if (part == 0 && block < p.lds) p.scale[row * p.lds + block] = (uint8_t)byte;
}

template <Elem T>
static hipError_t run_mx_quantize(MxRows p, hipStream_t stream) {
    const int64_t codes = p.ldq / 16, blocks = codes > p.lds ? codes : p.lds, most = (kMostLanes - 255) / 4 / blocks;   // rows a launch
    if (most < 1) return hipErrorInvalidValue;
    const unsigned magic = (unsigned)(((uint64_t)1 << 32) / blocks) + 1;       // (of one block: 2^32 and one more would not fit, but there are 16)
    for (int64_t left = p.M; left > 0;) {
        p.M = left < most ? left : most;
        const dim3 grid((unsigned)ceil_div(p.M * blocks * 4, 256));
        const hipError_t e = launch_kernel(kTimeSplitQuantize, p.chan_depth ? mx_quantize_kernel<T, true> : mx_quantize_kernel<T, false>, grid,
                                           dim3(256), 0, stream, p, (unsigned)blocks, magic);
        if (e != hipSuccess) return e;
        left -= p.M;
        p.X = static_cast<const elem_t<T>*>(p.X) + p.M * p.ldx;
        p.q += p.M * p.ldq;
        p.scale += p.M * p.lds;
    }
    return hipSuccess;
}

hipError_t launch_mx_quantize(const void* X, int type, int64_t ldx, int64_t M, int C, int g, int s, const int32_t* chan_src,
                              const int32_t* chan_depth, uint8_t* q, int64_t ldq, uint8_t* scale, int64_t lds, hipStream_t stream) {
    const MxRows p{X, ldx, M, C, g, s, chan_src, chan_depth, q, ldq, scale, lds};
    switch (static_cast<Elem>(type)) {
        case Elem::f32: return run_mx_quantize<Elem::f32>(p, stream);
        case Elem::bf16: return run_mx_quantize<Elem::bf16>(p, stream);
        case Elem::f16: return run_mx_quantize<Elem::f16>(p, stream);
    }
    return hipErrorInvalidValue;
}

struct MxValues {
    const uint8_t* q;
    int64_t ldq;
    const uint8_t* scale;
    int64_t lds, M;
    int cols;
    void* Y;
    int64_t ldy;
};

// One lane per 8 columns.
template <Elem OUT>
__global__ __launch_bounds__(256) void mx_values_kernel(MxValues p, unsigned eights) {
    const unsigned at = blockIdx.x * 256 + threadIdx.x;
    const int64_t row = at / eights;
    if (row >= p.M) return;
    const int k0 = (int)(at - (unsigned)row * eights) * 8;
    float v[8];
    mx_values8(*reinterpret_cast<const unsigned*>(p.q + row * p.ldq + k0 / 2), p.scale[row * p.lds + k0 / kMxBlock], v);
    elem_t<OUT>* y = static_cast<elem_t<OUT>*>(p.Y) + row * p.ldy + k0;
    elem_t<OUT> o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = float_to_elem<OUT>(v[e]);
    if (k0 + 8 <= p.cols) {
#pragma unroll
        for (int h = 0; h < 8 / kVec<OUT>; ++h) {
            elem_t<OUT> piece[kVec<OUT>];
#pragma unroll
            for (int e = 0; e < kVec<OUT>; ++e) piece[e] = o[h * kVec<OUT> + e];
            store_piece<OUT>(y + h * kVec<OUT>, piece);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (k0 + e < p.cols) y[e] = o[e];
    }
}

template <Elem OUT>
static hipError_t run_mx_values(MxValues p, hipStream_t stream) {
    const int64_t eights = ceil_div(p.cols, 8), most = (kMostLanes - 255) / eights;
    for (int64_t left = p.M; left > 0;) {
        p.M = left < most ? left : most;
        const hipError_t e = launch_kernel(0, mx_values_kernel<OUT>, dim3((unsigned)ceil_div(p.M * eights, 256)), dim3(256), 0, stream, p, (unsigned)eights);
        if (e != hipSuccess) return e;
        left -= p.M;
        p.q += p.M * p.ldq;
        p.scale += p.M * p.lds;
        p.Y = static_cast<elem_t<OUT>*>(p.Y) + p.M * p.ldy;
    }
    return hipSuccess;
}

hipError_t launch_mx_values(const uint8_t* q, int64_t ldq, const uint8_t* scale, int64_t lds, int64_t M, int64_t cols, void* Y, int out_type,
                            int64_t ldy, hipStream_t stream) {
    const MxValues p{q, ldq, scale, lds, M, (int)cols, Y, ldy};
    switch (static_cast<Elem>(out_type)) {
        case Elem::f32: return run_mx_values<Elem::f32>(p, stream);
        case Elem::bf16: return run_mx_values<Elem::bf16>(p, stream);
        case Elem::f16: return run_mx_values<Elem::f16>(p, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace ocs
