// Keys and values of tokens onto their grids as they are written into the pages of a cache, and back to numbers.
//
// A row is a token's D values of a head: k' = k * 2^-depth, then 8 bits (Eq. 1 on the row's own grid: T = max|k'|, step T / 127) or 4
// (blocks of 32 columns on powers of two).  A wave takes the rows of one token, so that it looks for the token's sequence once; 8 columns
// per lane, 4 to 32 lanes a row, the row's maximum by exchanges between them.  Bound by HBM
// for many tokens (34832 of 8 heads of 128 from 4 bits to bf16 39.7 us, 4.6 TB/s), by one launch for few (64 tokens 2.4 us).
#include "cache.h"

namespace ocs {

struct CacheRows {
    Cache c;
    Sequences s;
    void* K;
    int64_t ldk, hdk;
    void* V;
    int64_t ldv, hdv;
    int t0;                                     // first token of this launch
};

template <Elem T>
__device__ __forceinline__ void load8(const elem_t<T>* x, float (&v)[8]) {
#pragma unroll
    for (int h = 0; h < 8 / kVec<T>; ++h) {
        const u32x4 piece = load_piece<T>(x + h * kVec<T>);
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) v[h * kVec<T> + e] = piece_elem<T>(piece, e);
    }
}

template <Elem T>
__device__ __forceinline__ void store8(elem_t<T>* y, const float (&v)[8]) {
#pragma unroll
    for (int h = 0; h < 8 / kVec<T>; ++h) {
        elem_t<T> piece[kVec<T>];
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) piece[e] = float_to_elem<T>(v[h * kVec<T> + e]);
        store_piece<T>(y + h * kVec<T>, piece);
    }
}

// LANES lanes a row, 64 / LANES rows a wave at a time, TIMES times: rows 0 .. H - 1 of a token are its keys', H .. 2H - 1 its values'.
template <Elem T, CacheFormat F, int LANES, int TIMES, bool WRITE>
__global__ __launch_bounds__(256) void cache_rows_kernel(CacheRows p, unsigned waves_per_token) {
    constexpr int ROWS = 64 / LANES;
    const int lane = (int)threadIdx.x & 63, c = lane % LANES * 8, H = p.c.H, D = p.c.D;
    const unsigned wave = __builtin_amdgcn_readfirstlane(neighbours_on_an_xcd(blockIdx.x, gridDim.x) * 4 + (threadIdx.x >> 6));
    const unsigned nth = wave / waves_per_token, t = p.t0 + nth;
    if (t >= (unsigned)p.s.T) return;
    const int first = (int)(wave - nth * waves_per_token) * (ROWS * TIMES) + lane / LANES;
    int64_t position;
    const int b = sequence_of(p.s, (int)t, &position);
    if (b < 0) return;
    const int64_t row = cache_row(p.c, b, position);
    if (WRITE && row < 0) return;

    struct Row {
        bool live, values;
        int h;
        int64_t at;
    };
    auto row_of = [&](int i) {
        const int r = first + i * ROWS;
        Row w;
        w.live = r < 2 * H && c < D;
        w.values = r >= H;
        w.h = w.values ? r - H : r;
        w.at = row + (int64_t)w.h * p.c.P;
        return w;
    };
    auto elements = [&](const Row& w) {
        return w.values ? static_cast<elem_t<T>*>(p.V) + t * p.ldv + w.h * p.hdv + c : static_cast<elem_t<T>*>(p.K) + t * p.ldk + w.h * p.hdk + c;
    };
    auto scaled = [&](const Row& w, float (&v)[8], auto factor) {
        const int32_t* depth = w.values ? p.c.vdepth : p.c.kdepth;
        if (depth == nullptr) return;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= factor(depth[w.h * D + c + e]);
    };
    float v[TIMES][8];
    if constexpr (WRITE) {
#pragma unroll
        for (int i = 0; i < TIMES; ++i) {
            const Row w = row_of(i);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
            if (w.live) load8<T>(elements(w), v[i]);
        }
#pragma unroll
        for (int i = 0; i < TIMES; ++i) {
            const Row w = row_of(i);
            if (w.live) scaled(w, v[i], cache_halvings);
            unsigned big = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) big = mx_magnitude(v[i][e]) > big ? mx_magnitude(v[i][e]) : big;
            unsigned whole = big;                                 // of the row; 4 bits: `big` of the block of 4 lanes
#pragma unroll
            for (int m = 1; m < LANES; m *= 2) {
                const unsigned o = (unsigned)__shfl_xor((int)whole, m);
                whole = o > whole ? o : whole;
                if (m == 2) big = whole;
            }
            if (!w.live) continue;
            void* codes = w.values ? p.c.values : p.c.keys;
            void* scales = w.values ? p.c.vscales : p.c.kscales;
            if constexpr (F == CacheFormat::int8) {
                const float thr = __uint_as_float(whole), inv = inv_step_of(thr, 127.0f);
                unsigned q[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) q[e] = code_bits(v[i][e], inv, 127.0f);
                *reinterpret_cast<u32x2*>(static_cast<int8_t*>(codes) + w.at * D + c) = u32x2{pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7])};
                if (c == 0) static_cast<float*>(scales)[w.at] = __fdiv_rn(thr, 127.0f);
            } else {
                const bool finite = whole < 0x7F800000u;          // a row with NaN or an infinity: every scale 255
                const unsigned byte = finite ? mx_scale_byte(big) : 255u;
                *reinterpret_cast<unsigned*>(static_cast<uint8_t*>(codes) + w.at * (D / 2) + c / 2) = finite ? mx_codes8(v[i], mx_scale_value(byte)) : 0u;
                if (c % kMxBlock == 0) static_cast<uint8_t*>(scales)[w.at * (D / kMxBlock) + c / kMxBlock] = (uint8_t)byte;
            }
        }
    } else {
        u32x2 q[TIMES];
        float step[TIMES];
#pragma unroll
        for (int i = 0; i < TIMES; ++i) {
            const Row w = row_of(i);
            q[i] = u32x2{0u, 0u};
            step[i] = 0.0f;
            if (!w.live || row < 0) continue;                     // a position without a page: zeros
            const void* codes = w.values ? p.c.values : p.c.keys;
            const void* scales = w.values ? p.c.vscales : p.c.kscales;
            if constexpr (F == CacheFormat::int8) {
                q[i] = *reinterpret_cast<const u32x2*>(static_cast<const int8_t*>(codes) + w.at * D + c);
                step[i] = static_cast<const float*>(scales)[w.at];
            } else {
                q[i][0] = *reinterpret_cast<const unsigned*>(static_cast<const uint8_t*>(codes) + w.at * (D / 2) + c / 2);
                q[i][1] = static_cast<const uint8_t*>(scales)[w.at * (D / kMxBlock) + c / kMxBlock];
            }
        }
#pragma unroll
        for (int i = 0; i < TIMES; ++i) {
            const Row w = row_of(i);
            if (!w.live) continue;
            if constexpr (F == CacheFormat::int8) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = (float)(int8_t)(q[i][e / 4] >> (8 * (e % 4))) * step[i];
            } else {
                mx_values8(q[i][0], q[i][1], v[i]);
            }
            scaled(w, v[i], cache_doublings);
            store8<T>(elements(w), v[i]);
        }
    }
}

template <Elem T, CacheFormat F, bool WRITE>
static hipError_t run_cache_rows(CacheRows p, hipStream_t stream) {
    const int lanes = p.c.D <= 32 ? 4 : p.c.D <= 64 ? 8 : p.c.D <= 128 ? 16 : 32;
    // A token's rows by one wave, which looks its sequence and page up once for up to four times as many rows as it holds at a time; one time
    // each while there are fewer than 16 waves a compute unit (34832 tokens of 8 heads of 128 in 4 bits read as bf16, after 48 were written: one time each
    // 73 us, four 51; two tokens a wave gain nothing more).
    const int64_t at_once = ceil_div(2 * (int64_t)p.c.H, 64 / lanes), times = at_once * p.s.T >= 16 * compute_units() ? 4 : 1;
    const int64_t per_token = ceil_div(at_once, times), most = (kMostLanes / 64 - 3) / per_token;   // tokens a launch
    auto kernel = times == 1 ? cache_rows_kernel<T, F, 32, 1, WRITE> : cache_rows_kernel<T, F, 32, 4, WRITE>;
    if (lanes == 4) kernel = times == 1 ? cache_rows_kernel<T, F, 4, 1, WRITE> : cache_rows_kernel<T, F, 4, 4, WRITE>;
    if (lanes == 8) kernel = times == 1 ? cache_rows_kernel<T, F, 8, 1, WRITE> : cache_rows_kernel<T, F, 8, 4, WRITE>;
    if (lanes == 16) kernel = times == 1 ? cache_rows_kernel<T, F, 16, 1, WRITE> : cache_rows_kernel<T, F, 16, 4, WRITE>;
    for (int64_t t0 = 0; t0 < p.s.T; t0 += most) {
        const int64_t n = p.s.T - t0 < most ? p.s.T - t0 : most;
        p.t0 = (int)t0;
        const hipError_t e = launch_kernel(kTimeSplitQuantize, kernel, dim3((unsigned)ceil_div(n * per_token, 4)), dim3(256), 0, stream, p,
                                           (unsigned)per_token);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <Elem T>
static hipError_t run_cache_rows_of(const CacheRows& p, int format, bool write, hipStream_t stream) {
    if (format == (int)CacheFormat::int8)
        return write ? run_cache_rows<T, CacheFormat::int8, true>(p, stream) : run_cache_rows<T, CacheFormat::int8, false>(p, stream);
    return write ? run_cache_rows<T, CacheFormat::mx4, true>(p, stream) : run_cache_rows<T, CacheFormat::mx4, false>(p, stream);
}

hipError_t launch_cache_rows(bool write, void* K, int64_t ldk, int64_t hdk, void* V, int64_t ldv, int64_t hdv, int type, const Sequences& s,
                             int format, const Cache& c, hipStream_t stream) {
    const CacheRows p{c, s, K, ldk, hdk, V, ldv, hdv, 0};
    switch (static_cast<Elem>(type)) {
        case Elem::f32: return run_cache_rows_of<Elem::f32>(p, format, write, stream);
        case Elem::bf16: return run_cache_rows_of<Elem::bf16>(p, format, write, stream);
        case Elem::f16: return run_cache_rows_of<Elem::f16>(p, format, write, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace ocs
