// Product of operands on microscaled 4-bit grids: Y[m,n] = sum over k of x[m,k] w[n,k] + bias[n], where a block of 32 codes shares a power
// of two, on the matrix cores (v_mfma_scale_f32_16x16x128_f8f6f4, which takes codes and scale bytes as they are and adds in fp32).
//
// As in the int8 product with a scale per row the weights run down an accumulator tile and the tokens across it, and codes go from memory
// straight into LDS, 128 bytes (256 columns) of 8 rows per request, 16-byte chunks XOR-ed with the row.  A chunk is a block.  A row's 16
// scale bytes of two steps are a request of their own, one row per lane; a lane of quarter q takes chunks 2q and 2q + 1 of a step, so that
// their scales are two neighbouring bytes, which the instruction picks from one register.
// Many tokens: 8192 x 4096 x 4178 bf16 74 us, 3.8 PFLOP/s, 8192^3 4.2, where a bare loop of the instruction sustains 7.0; requests alone take
// 228 us of 270 on the latter, reads and products alone 221.  Few tokens: the weights' bytes, and the latency of one launch.
#include <type_traits>

#include "mx_grids.h"
#include "tile_requests.h"

namespace ocs {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct MxGemm {
    const uint8_t* Xq;
    int64_t ldx;
    const uint8_t* Xs;
    int64_t ldxs;
    const uint8_t* Wq;
    int64_t ldw;
    const uint8_t* Ws;
    int64_t ldws;
    int M, N, ksteps;                 // steps of 256 columns of K
    const float* bias;
    void* Y;
    int64_t ldy;
    int tiles_m, tiles_n;
};

// acc += a b over 128 columns; which byte of either scale register is a lane's block's
template <int BYTE_A, int BYTE_B>
__device__ __forceinline__ f32x4 mx_multiply(i32x4 a, i32x4 b, f32x4 acc, int scale_a, int scale_b) {
#if defined(__HIP_DEVICE_COMPILE__)
    const i32x8 wa = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1), wb = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, wb, acc, 4, 4, BYTE_A, scale_a, BYTE_B, scale_b);
#else
    (void)a;
    (void)b;
    (void)scale_a;
    (void)scale_b;
    return acc;
#endif
}

// A BM x BN tile (tokens x outputs) per workgroup, a ring of NBUF steps in LDS.
// ANY: pitches that are no multiples of 128, or so long that offsets inside a tile take 64 bits.
template <int BM, int BN, int WAVES_M, int WAVES_N, int NBUF, Elem OUT, bool ANY = false>
__global__ __launch_bounds__(WAVES_M * WAVES_N * 64) void mx_tile_kernel(MxGemm p) {
    constexpr int NW = WAVES_M * WAVES_N, ROWS = BM + BN;
    constexpr int XL = BM / 8 / NW, WL = BN / 8 / NW, LPS = XL + WL;
    constexpr int SL = (ROWS + 64 * NW - 1) / (64 * NW);              // requests of scales per wave, every second step
    constexpr int TM = BM / WAVES_M / 16, TN = BN / WAVES_N / 16;
    constexpr int STEP = ROWS * 128, SCALES = SL * NW * 1024, SBUF = NBUF / 2 + 1;
    static_assert(XL >= 1 && WL >= 1 && BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "whole requests per wave");
    static_assert(NBUF * (LPS + SL) < 64 && NBUF >= 2, "requests under way");
    __shared__ __align__(1024) int8_t lds[NBUF * STEP + SBUF * SCALES];
    const int tid = (int)threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WAVES_N, wn = wave % WAVES_N;
    int bm, bn;
    tile_of(blockIdx.x, p.tiles_m, p.tiles_n, &bm, &bn);
    const int row0 = bm * BM, col0 = bn * BN;

    // request u of a step: rows 8 (u NW + wave) + lane / 8 of the step's image, chunk slot lane % 8; first the rows of X, then those of W
    // (slot 4 h + q of a row holds chunk 2 q + h: at any time the matrix cores' reads are of neighbouring slots, in different banks)
    const int slot_of_row = (lane & 7) ^ (lane >> 3), piece = (slot_of_row & 3) * 2 + (slot_of_row >> 2);
    const int8_t* xbase = reinterpret_cast<const int8_t*>(p.Xq) + (int64_t)row0 * p.ldx;
    const int8_t* wbase = reinterpret_cast<const int8_t*>(p.Wq) + (int64_t)col0 * p.ldw;
    typename std::conditional<ANY, int64_t, unsigned>::type from[LPS];
#pragma unroll
    for (int u = 0; u < XL; ++u) {
        int r = (u * NW + wave) * 8 + (lane >> 3);
        r = row0 + r < p.M ? r : p.M - 1 - row0;
        from[u] = (decltype(from[0] + 0))(r * p.ldx + piece * 16);
    }
#pragma unroll
    for (int u = 0; u < WL; ++u) {
        int r = column_of<OUT>((u * NW + wave) * 8 + (lane >> 3));
        r = col0 + r < p.N ? r : p.N - 1 - col0;
        from[XL + u] = (decltype(from[0] + 0))(r * p.ldw + piece * 16);
    }
    // scales: row 64 (u NW + wave) + lane of the image (beyond its rows: the last one again)
    const int8_t* scales_from[SL];
#pragma unroll
    for (int u = 0; u < SL; ++u) {
        int r = (u * NW + wave) * 64 + lane;
        r = r < ROWS ? r : ROWS - 1;
        if (r < BM) {
            r = row0 + r < p.M ? row0 + r : p.M - 1;
            scales_from[u] = reinterpret_cast<const int8_t*>(p.Xs) + r * p.ldxs;
        } else {
            r = col0 + column_of<OUT>(r - BM);
            r = r < p.N ? r : p.N - 1;
            scales_from[u] = reinterpret_cast<const int8_t*>(p.Ws) + r * p.ldws;
        }
    }
    const unsigned lds0 = lds_address(lds) + (unsigned)wave * 1024;
    auto request = [&](int u, int kt, int buf) {
        const int at = buf * STEP + u * NW * 1024;
        const int8_t* base = (u < XL ? xbase : wbase) + (int64_t)kt * 128;
        if constexpr (ANY) {
            // A pitch that ends inside the last step: the lanes whose chunks are not there write zeros themselves.  (Every request has lanes
            // whose chunks are, so that requests under way can be counted.)
            if ((int64_t)kt * 128 + piece * 16 >= (u < XL ? p.ldx : p.ldw))
                *reinterpret_cast<i32x4*>(lds + at + wave * 1024 + lane * 16) = i32x4{0, 0, 0, 0};
            else
                request_1k(base + from[u], lds0 + (unsigned)at);
        } else {
            request_1k(base, from[u], lds0 + (unsigned)at);
        }
    };
    auto request_scales = [&](int kt) {                               // of steps kt and kt + 1, kt even
#pragma unroll
        for (int u = 0; u < SL; ++u)
            request_1k(scales_from[u] + (int64_t)kt * 8, lds0 + (unsigned)(NBUF * STEP + (kt >> 1) % SBUF * SCALES + u * NW * 1024));
    };

    f32x4 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int fr = lane & 15, fq = lane >> 4;
    i32x4 xf[2][TM], wf[TN];                                          // (the weights' of the next half take the place of those just multiplied)
    int xs[TM], next_xs[TM], ws[TN];                                  // scales of both halves of a step
    auto read_x = [&](int j, int buf, int ks) {
        const int slot = ((4 * ks + fq) ^ (fr & 7)) * 16;
        xf[ks][j] = *reinterpret_cast<const i32x4*>(lds + buf * STEP + (wm * (BM / WAVES_M) + fr) * 128 + slot + j * 2048);
    };
    auto read_w = [&](int i, int buf, int ks) {
        const int slot = ((4 * ks + fq) ^ (fr & 7)) * 16;
        wf[i] = *reinterpret_cast<const i32x4*>(lds + buf * STEP + BM * 128 + (wn * (BN / WAVES_N) + fr) * 128 + slot + i * 2048);
    };
    const int8_t* xs_at = lds + NBUF * STEP + (wm * (BM / WAVES_M) + fr) * 16 + 2 * fq;
    const int8_t* ws_at = lds + NBUF * STEP + (BM + wn * (BN / WAVES_N) + fr) * 16 + 2 * fq;
    auto scales_of = [&](int kt) { return (kt >> 1) % SBUF * SCALES + (kt & 1) * 8; };
    auto read_xs = [&](int j, int step_at) { next_xs[j] = *reinterpret_cast<const unsigned short*>(xs_at + step_at + j * 256); };
    auto read_ws = [&](int i, int step_at) { ws[i] = *reinterpret_cast<const unsigned short*>(ws_at + step_at + i * 256); };
    auto multiply = [&](int i, auto half) {
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = mx_multiply<half.value, half.value>(wf[i], xf[half.value][j], acc[i][j], ws[i], xs[j]);
        // here and not later: the compiler would deal these products over the whole step, and the operands into scratch memory
#pragma unroll
        for (int j = 0; j < TM; ++j) asm volatile("" : "+v"(acc[i][j]));
    };

    // Step kt: its first half and its scales are in registers when it begins; the second is read while the first is multiplied.  Then comes
    // the one barrier of a step: every wave's part of step kt + 1 has landed and every wave has read all of step kt, so that the requests of
    // step kt + NBUF go into its buffer, NBUF - 1 whole steps ahead of their use.
    constexpr int XPR = (TM + TN - 1) / TN, RPR = (LPS + TN - 1) / TN;
    const int steps = p.ksteps;
#pragma unroll
    for (int u = 0; u < NBUF; ++u)
        if (u < steps) {
            if (u % 2 == 0) request_scales(u);
#pragma unroll
            for (int f = 0; f < LPS; ++f) request(f, u, u);
        }
    // (the requests of the last step that may stay under way are counted without its scales, which come first: a wait too many at most)
    if (steps >= NBUF) wait_requests<(NBUF - 1) * LPS>();
    else wait_requests<0>();
    __syncthreads();
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        read_x(j, 0, 0);
        read_xs(j, 0);
    }
#pragma unroll
    for (int i = 0; i < TN; ++i) {
        read_w(i, 0, 0);
        read_ws(i, 0);
    }
    // MORE: there is a step kt + NBUF, and so kt + 1 (known in the loop over whole rings, looked up behind it)
    auto step = [&](int buf, int kt, auto known) {
        constexpr bool KNOWN = decltype(known)::value;
        const bool more = KNOWN || kt + NBUF < steps, next = KNOWN || kt + 1 < steps;
#pragma unroll
        for (int j = 0; j < TM; ++j) xs[j] = next_xs[j];
#pragma unroll
        for (int i = 0; i < TN; ++i) {
#pragma unroll
            for (int j = i * XPR; j < (i + 1) * XPR && j < TM; ++j) read_x(j, buf, 1);
            __builtin_amdgcn_sched_barrier(0);
            multiply(i, std::integral_constant<int, 0>{});
            __builtin_amdgcn_sched_barrier(0);
            read_w(i, buf, 1);
        }
        // every read of this step's buffer has returned
        __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
        if (KNOWN || kt + NBUF <= steps) wait_requests<(NBUF - 2) * LPS>();
        else wait_requests<0>();
        __syncthreads();
        if (more && ((kt + NBUF) & 1) == 0) request_scales(kt + NBUF);
        const int next_at = scales_of(kt + 1);
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            if (next) {
#pragma unroll
                for (int j = i * XPR; j < (i + 1) * XPR && j < TM; ++j) {
                    read_x(j, (buf + 1) % NBUF, 0);
                    read_xs(j, next_at);
                }
            }
            if (more) {
#pragma unroll
                for (int u = i * RPR; u < (i + 1) * RPR && u < LPS; ++u) request(u, kt + NBUF, buf);
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply(i, std::integral_constant<int, 1>{});
            __builtin_amdgcn_sched_barrier(0);
            if (next) {
                read_w(i, (buf + 1) % NBUF, 0);
                read_ws(i, next_at);
            }
        }
    };
    int kt = 0;
    for (; kt + 2 * NBUF <= steps; kt += NBUF) {
#pragma unroll
        for (int u = 0; u < NBUF; ++u) step(u, kt + u, std::true_type{});
    }
    for (; kt < steps; kt += NBUF) {
#pragma unroll
        for (int u = 0; u < NBUF; ++u)
            if (kt + u < steps) step(u, kt + u, std::false_type{});
    }

    // NV accumulator tiles make 16 bytes of a token's outputs
    constexpr int NV = OUT == Elem::f32 ? 1 : 2;
    const int n0 = col0 + wn * (BN / WAVES_N) + fq * 4 * NV, m0 = row0 + wm * (BM / WAVES_M) + fr;
    f32x4 bias[TN];
#pragma unroll
    for (int i = 0; i < TN; ++i) {
        bias[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (p.bias) bias[i] = four_of(p.bias, n0 + (i / NV) * 16 * NV + (i % NV) * 4, p.N);
    }
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        const int m = m0 + j * 16;
        if (m >= p.M) continue;
        elem_t<OUT>* y = static_cast<elem_t<OUT>*>(p.Y) + (int64_t)m * p.ldy + n0;
#pragma unroll
        for (int i = 0; i < TN; i += NV) {
            elem_t<OUT> v[4 * NV];
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * q + e] = float_to_elem<OUT>(acc[i + q][j][e] + bias[i + q][e]);
            if (n0 + i * 16 + 4 * NV <= p.N) {
                store_piece<OUT>(y + i * 16, v);
            } else {
#pragma unroll
                for (int e = 0; e < 4 * NV; ++e)
                    if (n0 + i * 16 + e < p.N) y[i * 16 + e] = v[e];
            }
        }
    }
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int NBUF, Elem OUT, bool ANY = false>
static hipError_t run_mx_tile(MxGemm p, hipStream_t stream) {
    p.tiles_m = (int)ceil_div(p.M, BM);
    p.tiles_n = (int)ceil_div(p.N, BN);
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n;
    if (total > 0x7FFFFFFF || p.ksteps < 1) return hipErrorInvalidValue;
    return launch_kernel(kTimeGemm, mx_tile_kernel<BM, BN, WAVES_M, WAVES_N, NBUF, OUT, ANY>, dim3((unsigned)total),
                         dim3(WAVES_M * WAVES_N * 64), 0, stream, p);
}

// Few tokens: 16 XT tokens and 16 WT outputs per workgroup, the steps of K dealt over its NW waves, whose sums meet in LDS in the order of
// the waves.  Each weight is used once, so codes and scales go from memory straight to the lanes that multiply them, a step ahead.
// IN: the tokens' codes in memory, or rows of X of that type: every workgroup puts all of them on their grids itself while its first weights
// are on their way, into LDS, and the workgroups share the writing of codes and scales to memory.
struct Codes {};
template <Elem T>
struct RowsOf {
    static constexpr Elem type = T;
};

// Bytes of LDS that a token's codes and scales take.
__host__ __device__ inline int mx_image_row(int ksteps) { return ksteps * 136 + 16; }

template <int XT, int WT, int NW, Elem OUT, typename IN>
__global__ __launch_bounds__(NW * 64) void mx_few_kernel(MxGemm p, MxRows rows) {
    constexpr bool GIVEN = std::is_same<IN, Codes>::value;
    constexpr int NT = NW * 64;
    __shared__ __align__(16) float sums[NW][XT * 16][WT * 16 + 4];
    extern __shared__ __align__(16) uint8_t image[];
    const int tid = (int)threadIdx.x, lane = tid & 63, fr = lane & 15, fq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col0 = (int)(blockIdx.x % (unsigned)p.tiles_n) * (WT * 16), row0 = (int)(blockIdx.x / (unsigned)p.tiles_n) * (XT * 16);
    const uint8_t* w[WT];
    const uint8_t* ws[WT];
#pragma unroll
    for (int i = 0; i < WT; ++i) {
        int n = col0 + i * 16 + fr;
        n = n < p.N ? n : p.N - 1;
        w[i] = p.Wq + n * p.ldw + 32 * fq;
        ws[i] = p.Ws + n * p.ldws + 2 * fq;
    }
    const uint8_t* x[XT];
    const uint8_t* xs[XT];
#pragma unroll
    for (int j = 0; j < XT; ++j) {
        const int m = row0 + j * 16 + fr, r = m < p.M ? m : p.M - 1;
        x[j] = GIVEN ? p.Xq + r * p.ldx + 32 * fq : image + r * mx_image_row(p.ksteps) + 32 * fq;
        xs[j] = GIVEN ? p.Xs + r * p.ldxs + 2 * fq : image + r * mx_image_row(p.ksteps) + p.ksteps * 128 + 2 * fq;
    }
    struct Operands {
        i32x4 w[2][WT], x[2][XT];
        int ws[WT], xs[XT];
    };
    auto chunk = [&](const uint8_t* at, int64_t k, int64_t ld) {     // behind the pitch: zeros
        i32x4 r = {0, 0, 0, 0};
        if (k + 32 * fq < ld) r = *reinterpret_cast<const i32x4*>(at + k);
        return r;
    };
    auto load = [&](int kt, Operands& o) {
        const int64_t k = (int64_t)kt * 128;
#pragma unroll
        for (int i = 0; i < WT; ++i) {
            o.ws[i] = *reinterpret_cast<const unsigned short*>(ws[i] + kt * 8);
#pragma unroll
            for (int h = 0; h < 2; ++h) o.w[h][i] = chunk(w[i], k + 16 * h, p.ldw);
        }
        if constexpr (GIVEN) {
#pragma unroll
            for (int j = 0; j < XT; ++j) {
                o.xs[j] = *reinterpret_cast<const unsigned short*>(xs[j] + kt * 8);
#pragma unroll
                for (int h = 0; h < 2; ++h) o.x[h][j] = chunk(x[j], k + 16 * h, p.ldx);
            }
        }
    };
    Operands next;
    if (wave < p.ksteps) load(wave, next);
    if constexpr (!GIVEN) {
        // four lanes a block, 8 columns each, as the pass over rows does it
        const int blocks = p.ksteps * 8, total = p.M * blocks, share = (total + (int)gridDim.x - 1) / (int)gridDim.x;
        const int mine = (int)blockIdx.x * share, pitch = mx_image_row(p.ksteps);
        for (int o = tid; o < total * 4; o += NT) {
            const int at = o >> 2, row = at / blocks, block = at - row * blocks, part = o & 3;
            const int k0 = block * kMxBlock + part * 8;
            float v[8];
            mx_expanded8<IN::type, false>(rows, static_cast<const elem_t<IN::type>*>(rows.X) + row * rows.ldx, k0, k0 < (rows.C + rows.s) * rows.g, v);
            unsigned big = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) big = mx_magnitude(v[e]) > big ? mx_magnitude(v[e]) : big;
            const unsigned byte = mx_scale_byte(quad_max(big));
            const unsigned codes = byte == 255u ? 0u : mx_codes8(v, mx_scale_value(byte));
            *reinterpret_cast<unsigned*>(image + row * pitch + block * 16 + part * 4) = codes;
            if (part == 0) image[row * pitch + p.ksteps * 128 + block] = (uint8_t)byte;
            if (at >= mine && at < mine + share) {
                if ((int64_t)block * 16 < rows.ldq) *reinterpret_cast<unsigned*>(rows.q + row * rows.ldq + block * 16 + part * 4) = codes;
                if (part == 0 && block < rows.lds) rows.scale[row * rows.lds + block] = (uint8_t)byte;
            }
        }
        // the padding behind the last step
        const int64_t code_pad = rows.ldq / 16 - blocks, scale_pad = rows.lds - blocks;
        for (int r = (int)blockIdx.x; r < p.M; r += (int)gridDim.x) {
            for (int64_t o = tid; o < code_pad; o += NT) *reinterpret_cast<i32x4*>(rows.q + r * rows.ldq + (blocks + o) * 16) = i32x4{0, 0, 0, 0};
            for (int64_t o = tid; o < scale_pad; o += NT) rows.scale[r * rows.lds + blocks + o] = 0;
        }
        __syncthreads();
    }
    f32x4 acc[WT][XT];
#pragma unroll
    for (int i = 0; i < WT; ++i)
#pragma unroll
        for (int j = 0; j < XT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int kt = wave; kt < p.ksteps; kt += NW) {
        Operands o = next;
        if (kt + NW < p.ksteps) load(kt + NW, next);
        if constexpr (!GIVEN) {                               // (rows of tokens that are not there repeat the last one's)
#pragma unroll
            for (int j = 0; j < XT; ++j) {
                o.xs[j] = *reinterpret_cast<const unsigned short*>(xs[j] + kt * 8);
#pragma unroll
                for (int h = 0; h < 2; ++h) o.x[h][j] = *reinterpret_cast<const i32x4*>(x[j] + kt * 128 + 16 * h);
            }
        }
#pragma unroll
        for (int i = 0; i < WT; ++i)
#pragma unroll
            for (int j = 0; j < XT; ++j) {
                acc[i][j] = mx_multiply<0, 0>(o.w[0][i], o.x[0][j], acc[i][j], o.ws[i], o.xs[j]);
                acc[i][j] = mx_multiply<1, 1>(o.w[1][i], o.x[1][j], acc[i][j], o.ws[i], o.xs[j]);
            }
    }
#pragma unroll
    for (int i = 0; i < WT; ++i)
#pragma unroll
        for (int j = 0; j < XT; ++j) *reinterpret_cast<f32x4*>(&sums[wave][j * 16 + fr][i * 16 + fq * 4]) = acc[i][j];
    __syncthreads();
    for (int o = tid; o < XT * 16 * WT * 16; o += NT) {
        const int t = o / (WT * 16), c = o % (WT * 16), mm = row0 + t, n = col0 + c;
        if (mm >= p.M || n >= p.N) continue;
        float v = sums[0][t][c];
#pragma unroll
        for (int q = 1; q < NW; ++q) v += sums[q][t][c];
        if (p.bias) v += p.bias[n];
        static_cast<elem_t<OUT>*>(p.Y)[(int64_t)mm * p.ldy + n] = float_to_elem<OUT>(v);
    }
}

template <int XT, int WT, int NW, Elem OUT, typename IN>
static hipError_t run_mx_few(MxGemm p, const MxRows& rows, hipStream_t stream) {
    p.tiles_m = (int)ceil_div(p.M, XT * 16);
    p.tiles_n = (int)ceil_div(p.N, WT * 16);
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n;
    if (total > 0x7FFFFFFF || p.ksteps < 1) return hipErrorInvalidValue;
    const unsigned lds = std::is_same<IN, Codes>::value ? 0u : (unsigned)(p.M * mx_image_row(p.ksteps));
    return launch_kernel(kTimeGemm, mx_few_kernel<XT, WT, NW, OUT, IN>, dim3((unsigned)total), dim3(NW * 64), lds, stream, p, rows);
}

// The kernel by shape.
//
// Up to 32 tokens, or while 64 x 16 tiles are no more than the compute units: K over a workgroup's waves, 16 outputs a workgroup, or 32
// where 16 make more workgroups than compute units (us from a graph, 16 / 32: 1 x 4096 x 4096 4.3 / 5.9, 1 x 6000 x 3150 5.3 / 5.1,
// 16 x 6000 x 3150 6.8 / 5.9, 20 x 6000 x 3150 7.7 / 6.8).
// Then tiles: rounds of the chip times what a tile takes, a constant and a cost per step in 10 ns, fitted to these (us, bf16 outputs,
// three sets of operands in turn, 256 x 256 / 128 x 128, 64 x 128 and 64 x 64 two to a unit):
//   8192 x 4096 x 4178    78.7 /  95.7 / 124.3 / 183.8       700 x 6000 x 3150    24.5 / 17.9 / 22.1 / 27.6
//   8192 x 8192 x 8192   259.4 / 339.2 / 467.7 / 634.8       333 x 2049 x 1052    23.7 /  9.1 /  6.7 /  6.9
//   4096 x 4096 x 4096    40.2 /  46.8 /  57.7 /  90.7       700 x 33001 x 1575   48.6 / 47.8 / 49.4 / 78.7
template <Elem OUT>
static hipError_t run_mx_gemm(const MxGemm& p, hipStream_t stream) {
    const int64_t cus = compute_units();
    const bool wide = ceil_div(p.N, 16) > cus;
    if (p.M <= 16) return wide ? run_mx_few<1, 2, 8, OUT, Codes>(p, MxRows{}, stream) : run_mx_few<1, 1, 8, OUT, Codes>(p, MxRows{}, stream);
    if (p.M <= 32) return wide ? run_mx_few<2, 2, 8, OUT, Codes>(p, MxRows{}, stream) : run_mx_few<2, 1, 8, OUT, Codes>(p, MxRows{}, stream);
    if (ceil_div(p.M, 64) * ceil_div(p.N, 16) <= cus) return run_mx_few<4, 1, 8, OUT, Codes>(p, MxRows{}, stream);
    if (p.ldx >= kWidePitch || p.ldw >= kWidePitch || p.ldx % 128 != 0 || p.ldw % 128 != 0) return run_mx_tile<64, 64, 2, 2, 4, OUT, true>(p, stream);
    const auto cost = [&](int64_t bm, int64_t bn, int64_t at_once, int64_t fixed, int64_t step) {
        return ceil_div(ceil_div(p.M, bm) * ceil_div(p.N, bn), at_once * cus) * (fixed + step * p.ksteps);
    };
    const int64_t by_tile[4] = {cost(64, 64, 2, 250, 53), cost(64, 128, 2, 200, 92), cost(128, 128, 2, 450, 116), cost(256, 256, 1, 1350, 150)};
    int best = 0;
    for (int i = 1; i < 4; ++i)
        if (by_tile[i] < by_tile[best]) best = i;
    switch (best) {
        case 0: return run_mx_tile<64, 64, 2, 2, 4, OUT>(p, stream);
        case 1: return run_mx_tile<64, 128, 2, 4, 2, OUT>(p, stream);
        case 2: return run_mx_tile<128, 128, 2, 4, 2, OUT>(p, stream);
        default: return run_mx_tile<256, 256, 4, 2, 2, OUT>(p, stream);
    }
}

// Outputs by the launch, as in the int8 product: as a rule all of them.
template <Elem OUT>
static hipError_t run_mx_ranges(const MxGemm& p, int64_t M, int64_t N, hipStream_t stream) {
    constexpr int64_t kMostRows = (int64_t)1 << 28, kMostColumns = (int64_t)1 << 26, kMostOutputs = (int64_t)1 << 35;
    for (int64_t n0 = 0; n0 < N; n0 += kMostColumns) {
        const int64_t cols = N - n0 < kMostColumns ? N - n0 : kMostColumns;
        const int64_t most = kMostOutputs / cols < kMostRows ? kMostOutputs / cols : kMostRows;
        for (int64_t m0 = 0; m0 < M; m0 += most) {
            MxGemm q = p;
            q.M = (int)(M - m0 < most ? M - m0 : most);
            q.N = (int)cols;
            q.Xq += m0 * p.ldx;
            q.Xs += m0 * p.ldxs;
            q.Wq += n0 * p.ldw;
            q.Ws += n0 * p.ldws;
            if (p.bias) q.bias += n0;
            q.Y = static_cast<elem_t<OUT>*>(p.Y) + m0 * p.ldy + n0;
            const hipError_t e = run_mx_gemm<OUT>(q, stream);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

hipError_t launch_qgemm_mx(const uint8_t* Xq, int64_t ldx, const uint8_t* Xs, int64_t ldxs, const uint8_t* Wq, int64_t ldw,
                           const uint8_t* Ws, int64_t ldws, int64_t M, int64_t N, int64_t Kexp, const float* bias, void* Y, int out_type,
                           int64_t ldy, hipStream_t stream) {
    const MxGemm p{Xq, ldx, Xs, ldxs, Wq, ldw, Ws, ldws, 0, 0, (int)ceil_div(Kexp, 256), bias, Y, ldy, 0, 0};
    switch (static_cast<Elem>(out_type)) {
        case Elem::f32: return run_mx_ranges<Elem::f32>(p, M, N, stream);
        case Elem::bf16: return run_mx_ranges<Elem::bf16>(p, M, N, stream);
        case Elem::f16: return run_mx_ranges<Elem::f16>(p, M, N, stream);
    }
    return hipErrorInvalidValue;
}

// 16 waves share the pass over the rows and K while every workgroup has a compute unit to itself, 8 where there are more (us, 8 waves / 16:
// 1 x 3000 -> 6000 6.7 / 6.1, 1 x 4096 -> 4096 6.8 / 6.0, 16 x 250 -> 4000 6.1 / 5.1, 1 x 4096 -> 12000 9.6 / 12.1).
template <Elem OUT, typename IN>
static hipError_t run_forward_mx(const MxGemm& p, const MxRows& rows, hipStream_t stream) {
    const int64_t cus = compute_units();
    if (ceil_div(p.N, 16) <= cus) return run_mx_few<1, 1, 16, OUT, IN>(p, rows, stream);
    if (ceil_div(p.N, 32) <= cus) return run_mx_few<1, 2, 16, OUT, IN>(p, rows, stream);
    return run_mx_few<1, 2, 8, OUT, IN>(p, rows, stream);
}

template <Elem OUT>
static hipError_t run_forward_mx_of(const MxGemm& p, const MxRows& rows, int type, hipStream_t stream) {
    switch (static_cast<Elem>(type)) {
        case Elem::f32: return run_forward_mx<OUT, RowsOf<Elem::f32>>(p, rows, stream);
        case Elem::bf16: return run_forward_mx<OUT, RowsOf<Elem::bf16>>(p, rows, stream);
        case Elem::f16: return run_forward_mx<OUT, RowsOf<Elem::f16>>(p, rows, stream);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_forward_mx(const void* X, int type, int64_t ldx, int64_t M, int C, int g, int s, const int32_t* chan_src, uint8_t* Xq,
                             int64_t ldq, uint8_t* Xs, int64_t ldxs, const uint8_t* Wq, int64_t ldw, const uint8_t* Ws, int64_t ldws,
                             int64_t N, const float* bias, void* Y, int out_type, int64_t ldy, bool apart, hipStream_t stream) {
    const int64_t Kexp = (int64_t)(C + s) * g;
    // One launch while every workgroup's pass over all rows takes its lanes two rounds at most; beyond, that costs more than a launch of its own
    // (us, calls one after the other, one launch / two: 1 x 250 -> 4000 4.0 / 6.5, 1 x 3000 -> 6000 6.7 / 8.0, 2 x 3000 -> 6000 7.4 / 8.2, 1 x 4096 ->
    // 12000 10.1 / 12.5; 4 x 3000 -> 6000 8.6 / 8.5, 8 x 1000 -> 4000 7.7 / 6.5, 16 x 3000 -> 6000 17.9 / 9.1), nor with more than two workgroups
    // a compute unit, which repeat it one after the other (1 x 1500 -> 33001 14.6 / 12.7).  It reads X and W while outputs are being written.
    if (apart && M <= 16 && M * ceil_div(Kexp, 256) <= 32 && ceil_div(N, 32) <= 2 * (int64_t)compute_units()) {
        const MxGemm p{Xq, ldq, Xs, ldxs, Wq, ldw, Ws, ldws, (int)M, (int)N, (int)ceil_div(Kexp, 256), bias, Y, ldy, 0, 0};
        const MxRows rows{X, ldx, M, C, g, s, chan_src, nullptr, Xq, ldq, Xs, ldxs};
        switch (static_cast<Elem>(out_type)) {
            case Elem::f32: return run_forward_mx_of<Elem::f32>(p, rows, type, stream);
            case Elem::bf16: return run_forward_mx_of<Elem::bf16>(p, rows, type, stream);
            case Elem::f16: return run_forward_mx_of<Elem::f16>(p, rows, type, stream);
        }
    }
    const hipError_t e = launch_mx_quantize(X, type, ldx, M, C, g, s, chan_src, nullptr, Xq, ldq, Xs, ldxs, stream);
    if (e != hipSuccess) return e;
    return launch_qgemm_mx(Xq, ldq, Xs, ldxs, Wq, ldw, Ws, ldws, M, N, Kexp, bias, Y, out_type, ldy, stream);
}

}  // namespace ocs
