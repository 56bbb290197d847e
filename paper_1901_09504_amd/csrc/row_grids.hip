// Splitting and quantization with a grid per row: Eq. 1 with T taken over one row (a token of X, an output channel of W)
// of the expanded tensor.
//
// A row is read once: its values wait in registers for the row's maximum, then become codes.  A wave takes a short row, a
// workgroup a longer one; a row beyond what a workgroup's registers hold is read twice.  Bound by HBM for many rows (a row's
// elements in, a byte per expanded column out: 4096 x 4096 bf16 11.0 us, 4.6 TB/s) and by latency for few (20 x 3000 fp32 2.6 us).
// Rows with halvings (weights, once per layer) are bound by the look-up of a channel's factor, twice per element: 6000 x 3000 fp32 with
// 150 splits 53 us, without halvings 18.6.
#include "row_grids.h"

namespace ocs {

// The largest word over the NT lanes of a row (64: the wave, otherwise the workgroup).
template <int NT>
__device__ __forceinline__ unsigned row_max(unsigned v, unsigned* red) {
    v = wave_umax32(v);
    if constexpr (NT == 64) return v;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    unsigned m = red[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) m = red[w] > m ? red[w] : m;
    return m;
}

template <int NT>
__device__ __forceinline__ void row_barrier() {
    if constexpr (NT == 64) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
    } else {
        __syncthreads();
    }
}

// Bytes of LDS for a row's codes: whole pieces.
static int64_t image_bytes(int64_t K) { return round_up(K, 16); }

// Lanes of a workgroup: of four rows or of one.
template <int NT>
constexpr int kRowLanes = NT == 64 ? 256 : NT;

// NT lanes per row, U 16-byte pieces per lane: rows of up to NT * U pieces.  SCALED: 2^-chan_depth applies.
// Codes of whole pieces go straight to memory and into the row's image in LDS; what lies behind them (a last partial
// piece, the copies, the padding) is put together from the image, or with SCALED from the row again.
template <Elem T, int NT, int U, bool SCALED>
__global__ __launch_bounds__(kRowLanes<NT>) void row_grid_kernel(RowGrids p) {
    constexpr int VEC = kVec<T>, ROWS = kRowLanes<NT> / NT;
    __shared__ unsigned red[kRowLanes<NT> / 64];
    extern __shared__ __align__(16) int8_t images[];
    const int K = p.C * p.g, Ke = (p.C + p.s) * p.g;
    const int t = (int)threadIdx.x % NT;
    const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / NT;
    if (row >= p.M) return;                               // NT == 64: whole waves; otherwise never
    int8_t* image = images + (threadIdx.x / NT) * ((K + 15) & ~15);
    const elem_t<T>* x = static_cast<const elem_t<T>*>(p.X) + row * p.ldx;
    int8_t* q = p.Xq + row * p.ldq;
    const int pieces = K / VEC, rest = K % VEC;

    const int tail0 = pieces * VEC;
    FourSources first = four_sources(p, tail0 + 4 * t, K, Ke);      // of this lane's first word behind the pieces
    u32x4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = u * NT + t;
        raw[u] = u32x4{0u, 0u, 0u, 0u};
        if (i < pieces) raw[u] = load_piece<T>(x + i * VEC);
        else if (i == pieces && rest) raw[u] = load_partial<T>(x + i * VEC, rest);
    }
    auto value = [&](int u, int e) {
        float v = piece_elem<T>(raw[u], e);
        if constexpr (SCALED) {
            const int k = (u * NT + t) * VEC + e;
            if (k < K) v *= depth_factor(p, p.g == 1 ? k : k / p.g);
        }
        return v;
    };
    unsigned big = 0;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const unsigned m = magnitude(value(u, e));
            big = m > big ? m : big;
        }
    if constexpr (SCALED) {                               // a copy may carry fewer halvings than its source
        for (int k = K + t; k < Ke; k += NT) {
            int j;
            const int src = source_column(p, k, &j);
            const unsigned m = magnitude(elem_to_float<T>(x[src]) * depth_factor(p, j));
            big = m > big ? m : big;
        }
    }
    const float thr = p.clip * __uint_as_float(row_max<NT>(big, red));
    const float inv = inv_step_of(thr, p.qmax);
    if (t == 0) p.step[row] = __fdiv_rn(thr, p.qmax);

#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = u * NT + t;
        unsigned code[VEC / 4];
#pragma unroll
        for (int d = 0; d < VEC / 4; ++d)
            code[d] = pack4(code_bits(value(u, 4 * d), inv, p.qmax), code_bits(value(u, 4 * d + 1), inv, p.qmax),
                            code_bits(value(u, 4 * d + 2), inv, p.qmax), code_bits(value(u, 4 * d + 3), inv, p.qmax));
        if (i < pieces + (rest ? 1 : 0)) {
            unsigned* at = reinterpret_cast<unsigned*>(image + i * VEC);
            unsigned* to = reinterpret_cast<unsigned*>(q + i * VEC);
#pragma unroll
            for (int d = 0; d < VEC / 4; ++d) {
                at[d] = code[d];
                if (i < pieces) to[d] = code[d];
            }
        }
    }
    row_barrier<NT>();
    for (int k0 = tail0 + 4 * t; k0 < (int)p.ldq; k0 += 4 * NT) {
        const FourSources f = k0 == tail0 + 4 * t ? first : four_sources(p, k0, K, Ke);
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (SCALED) {
#pragma unroll
            for (int b = 0; b < 4; ++b)
                if (k0 + b >= K && k0 + b < Ke) v[b] = elem_to_float<T>(x[f.src[b]]) * depth_factor(p, f.channel[b]);
        }
        unsigned word = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            if (k0 + b >= Ke) continue;
            unsigned byte = (unsigned char)image[k0 + b < K || !SCALED ? f.src[b] : 0];
            if (SCALED && k0 + b >= K) byte = code_bits(v[b], inv, p.qmax) & 0xFFu;
            word |= byte << (8 * b);
        }
        *reinterpret_cast<unsigned*>(q + k0) = word;
    }
}

// Rows beyond the registers of a workgroup: the maximum first, then the row again (from the caches as far as they hold it).
template <Elem T, bool SCALED>
__global__ __launch_bounds__(256) void row_grid_long_kernel(RowGrids p) {
    constexpr int VEC = kVec<T>;
    __shared__ unsigned red[4];
    const int64_t K = (int64_t)p.C * p.g, Ke = (int64_t)(p.C + p.s) * p.g;
    const int t = (int)threadIdx.x;
    const int64_t row = blockIdx.x;
    const elem_t<T>* x = static_cast<const elem_t<T>*>(p.X) + row * p.ldx;
    int8_t* q = p.Xq + row * p.ldq;
    const int64_t pieces = K / VEC;
    auto at = [&](int64_t k) {                            // expanded column k
        float v;
        if (k < K) {
            v = elem_to_float<T>(x[k]);
            if constexpr (SCALED) v *= depth_factor(p, (int)(k / p.g));
        } else {
            int j;
            v = elem_to_float<T>(x[source_column(p, (int)k, &j)]);
            if constexpr (SCALED) v *= depth_factor(p, j);
        }
        return v;
    };
    unsigned big = 0;
    for (int64_t i = t; i < pieces; i += 256) {
        const u32x4 raw = load_piece<T>(x + i * VEC);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            float v = piece_elem<T>(raw, e);
            if constexpr (SCALED) v *= depth_factor(p, (int)((i * VEC + e) / p.g));
            const unsigned m = magnitude(v);
            big = m > big ? m : big;
        }
    }
    for (int64_t k = pieces * VEC + t; k < (SCALED ? Ke : K); k += 256) {
        const unsigned m = magnitude(at(k));
        big = m > big ? m : big;
    }
    const float thr = p.clip * __uint_as_float(row_max<256>(big, red));
    const float inv = inv_step_of(thr, p.qmax);
    if (t == 0) p.step[row] = __fdiv_rn(thr, p.qmax);
    for (int64_t i = t; i < pieces; i += 256) {
        const u32x4 raw = load_piece<T>(x + i * VEC);
        unsigned* to = reinterpret_cast<unsigned*>(q + i * VEC);
#pragma unroll
        for (int d = 0; d < VEC / 4; ++d) {
            unsigned c[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float v = piece_elem<T>(raw, 4 * d + e);
                if constexpr (SCALED) v *= depth_factor(p, (int)((i * VEC + 4 * d + e) / p.g));
                c[e] = code_bits(v, inv, p.qmax);
            }
            to[d] = pack4(c[0], c[1], c[2], c[3]);
        }
    }
    for (int64_t k0 = pieces * VEC + 4 * t; k0 < p.ldq; k0 += 4 * 256) {
        unsigned word = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b)
            if (k0 + b < Ke) word |= (code_bits(at(k0 + b), inv, p.qmax) & 0xFFu) << (8 * b);
        *reinterpret_cast<unsigned*>(q + k0) = word;
    }
}

// One launch for every `lanes` lanes' worth of rows, `rows` rows a workgroup: as a rule all of them.
template <Elem T, typename F>
static hipError_t launch_by_rows(RowGrids p, int lanes, int rows, F kernel, unsigned lds, hipStream_t stream) {
    const int64_t most = kMostLanes / lanes * rows;
    for (int64_t left = p.M; left > 0;) {
        p.M = left < most ? left : most;
        const hipError_t e = launch_kernel(kTimeSplitQuantize, kernel, dim3((unsigned)ceil_div(p.M, rows)), dim3((unsigned)lanes), lds, stream, p);
        if (e != hipSuccess) return e;
        left -= p.M;
        p.X = static_cast<const elem_t<T>*>(p.X) + p.M * p.ldx;
        p.Xq += p.M * p.ldq;
        p.step += p.M;
    }
    return hipSuccess;
}

template <Elem T, int NT, int U>
static hipError_t run_row_grids(const RowGrids& p, hipStream_t stream) {
    constexpr int LANES = kRowLanes<NT>, ROWS = LANES / NT;
    const unsigned lds = (unsigned)(image_bytes((int64_t)p.C * p.g) * ROWS);
    return launch_by_rows<T>(p, LANES, ROWS, p.chan_depth ? row_grid_kernel<T, NT, U, true> : row_grid_kernel<T, NT, U, false>, lds, stream);
}

template <Elem T>
static hipError_t run_row_grids_of(const RowGrids& p, hipStream_t stream) {
    const int64_t K = (int64_t)p.C * p.g, pieces = ceil_div(K, kVec<T>);
    if (p.ldq <= 0x7FFFF000) {                            // (a row's 32-bit column passes its end by one round of the workgroup)
        // A wave per row while two pieces a lane hold it, then a workgroup.  While every row can have a compute unit to itself, with as
        // many lanes as its pieces ask for: a lane's pieces are the latency (us, fp32, 256 lanes / 512 / 1024: 20 x 1500 2.8 / 2.55 / 2.56,
        // 20 x 3000 3.0 / 2.8 / 2.6, 256 x 6000 5.4 / 4.3 / 4.1).  With more rows, several workgroups a unit hide it instead, and fewer
        // lanes wait at a barrier (700 x 3000 4.75 / 4.7 / 5.8, 700 x 4096 6.5 / 5.8 / 7.1, 4096 x 1500 8.2 / 10.1 / 16.8, 4096 x 3000 12.5 / 13.7 /
        // 18.1, 4096 x 6000 27.1 / 24.9 / 30.9).
        const int64_t cus = compute_units();
        if (pieces <= 64) return run_row_grids<T, 64, 1>(p, stream);
        if (pieces <= 128) return run_row_grids<T, 64, 2>(p, stream);
        if (pieces <= 256) return run_row_grids<T, 256, 1>(p, stream);
        if (pieces <= 512) return p.M <= cus ? run_row_grids<T, 512, 1>(p, stream) : run_row_grids<T, 256, 2>(p, stream);
        if (pieces <= 1024) {
            if (p.M <= cus) return run_row_grids<T, 1024, 1>(p, stream);
            return p.M <= 4 * cus ? run_row_grids<T, 512, 2>(p, stream) : run_row_grids<T, 256, 4>(p, stream);
        }
        if (pieces <= 2048) return p.M <= cus ? run_row_grids<T, 1024, 2>(p, stream) : run_row_grids<T, 512, 4>(p, stream);
    }
    return launch_by_rows<T>(p, 256, 1, p.chan_depth ? row_grid_long_kernel<T, true> : row_grid_long_kernel<T, false>, 0, stream);
}

hipError_t launch_row_grids(const void* X, int type, int64_t ldx, int64_t M, int C, int g, int s, const int32_t* chan_src,
                            const int32_t* chan_depth, float clip, float qmax, int8_t* Xq, int64_t ldq, float* step,
                            hipStream_t stream) {
    const RowGrids p{X, ldx, M, C, g, s, chan_src, chan_depth, clip, qmax, Xq, ldq, step};
    switch (static_cast<Elem>(type)) {
        case Elem::f32: return run_row_grids_of<Elem::f32>(p, stream);
        case Elem::bf16: return run_row_grids_of<Elem::bf16>(p, stream);
        case Elem::f16: return run_row_grids_of<Elem::f16>(p, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace ocs
