// int8 product with a scale per row of either operand: Y[m,n] = acc * (step_x[m] * step_w[n]) + bias[n], acc exact in int32
// on the matrix cores (v_mfma_i32_16x16x64_i8).
//
// The weights are the matrix operand that runs down an accumulator tile and the tokens the one that runs across it: a lane then
// holds four consecutive outputs of one token and stores them as they are, without a detour through LDS.
// Codes go from memory straight into LDS, 128 bytes (one line) of 8 rows per request, 16-byte chunks XOR-ed with the row so that
// the matrix cores' reads of consecutive rows fall into different banks.
// Many tokens: 8192 x 4096 x 4178 bf16 118 us, 2.4 POPS, where a bare loop of these instructions on random codes sustains 4.1; a step's requests, LDS
// reads and products add up more than they hide (768 x 8192 -> 6016: 32 us of requests and 32 of products make 49).  Few tokens: the weights' bytes.
#include <type_traits>

#include "row_grids.h"
#include "tile_requests.h"

namespace ocs {

struct RowsGemm {
    const int8_t* Xq;
    int64_t ldx;
    const int8_t* Wq;
    int64_t ldw;
    int M, N, ksteps;                 // steps of 128 bytes of K
    const float* step_x;
    const float* step_w;
    const float* bias;
    void* Y;
    int64_t ldy;
    int tiles_m, tiles_n;
};

// A BM x BN tile (tokens x outputs) per workgroup, a ring of NBUF steps in LDS.
// WIDE: pitches of 2^24 bytes and more, whose offsets inside a tile do not fit 32 bits.
template <int BM, int BN, int WAVES_M, int WAVES_N, int NBUF, Elem OUT, bool WIDE = false>
__global__ __launch_bounds__(WAVES_M * WAVES_N * 64) void rows_tile_kernel(RowsGemm p) {
    constexpr int NW = WAVES_M * WAVES_N;
    constexpr int XL = BM / 8 / NW, WL = BN / 8 / NW, LPS = XL + WL;
    constexpr int TM = BM / WAVES_M / 16, TN = BN / WAVES_N / 16;
    constexpr int STEP = (BM + BN) * 128;
    static_assert(XL >= 1 && WL >= 1 && BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "whole requests per wave");
    static_assert(NBUF * LPS < 64 && NBUF >= 2, "requests under way");
    __shared__ __align__(1024) int8_t lds[NBUF * STEP];
    const int tid = (int)threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WAVES_N, wn = wave % WAVES_N;
    int bm, bn;
    tile_of(blockIdx.x, p.tiles_m, p.tiles_n, &bm, &bn);
    const int row0 = bm * BM, col0 = bn * BN;

    // request u of a step: rows 8 (u NW + wave) + lane / 8 of the step's image, chunk slot lane % 8; first the rows of X, then those of W
    const int piece = (lane & 7) ^ (lane >> 3);
    const int8_t* xbase = p.Xq + (int64_t)row0 * p.ldx;
    const int8_t* wbase = p.Wq + (int64_t)col0 * p.ldw;
    typename std::conditional<WIDE, int64_t, unsigned>::type from[LPS];
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
    const unsigned lds0 = lds_address(lds) + (unsigned)wave * 1024;
    const bool cut = p.ldx < (int64_t)p.ksteps * 128 || p.ldw < (int64_t)p.ksteps * 128;   // a pitch that ends inside the last step
    auto request = [&](int u, int kt, int buf) {
        const unsigned to = lds0 + (unsigned)(buf * STEP + u * NW * 1024);
        const int8_t* base = (u < XL ? xbase : wbase) + (int64_t)kt * 128;
        if (cut && kt == p.ksteps - 1)
            request_1k((int64_t)kt * 128 + piece * 16 < (u < XL ? p.ldx : p.ldw) ? base + from[u] : rows_zero_chunk, to);
        else if constexpr (WIDE)
            request_1k(base + from[u], to);
        else
            request_1k(base, from[u], to);
    };
    auto fetch = [&](int kt, int buf) {
#pragma unroll
        for (int u = 0; u < LPS; ++u) request(u, kt, buf);
    };

    i32x4 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    const int fr = lane & 15, fq = lane >> 4;
    i32x4 xf[2][TM], wf[2][TN];
    // fragment f of a half step: the token tiles first, then the weight tiles
    auto read = [&](int f, int buf, int ks) {
        const int slot = ((ks * 4 + fq) ^ (fr & 7)) * 16;
        if (f < TM)
            xf[ks][f] = *reinterpret_cast<const i32x4*>(lds + buf * STEP + (wm * (BM / WAVES_M) + fr) * 128 + slot + f * 2048);
        else
            wf[ks][f - TM] = *reinterpret_cast<const i32x4*>(lds + buf * STEP + BM * 128 + (wn * (BN / WAVES_N) + fr) * 128 + slot +
                                                             (f - TM) * 2048);
    };
    auto multiply = [&](int i, int ks) {
#pragma unroll
        for (int j = 0; j < TM; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[ks][i], xf[ks][j], acc[i][j], 0, 0, 0);
    };

    // Step kt: its first half is in registers when it begins; the second is read while the first is multiplied.  Then comes the
    // one barrier of a step: every wave's part of step kt + 1 has landed and every wave has read all of step kt, so that the requests of
    // step kt + NBUF go into its buffer, NBUF - 1 whole steps ahead of their use.  Reads and requests are dealt over the rows of
    // products: the matrix cores run on while they are issued.
    constexpr int FR = TM + TN, FPR = (FR + TN - 1) / TN, RPR = (LPS + TN - 1) / TN;
    const int steps = p.ksteps;
#pragma unroll
    for (int u = 0; u < NBUF; ++u)
        if (u < steps) fetch(u, u);
    if (steps >= NBUF) wait_requests<(NBUF - 1) * LPS>();
    else wait_requests<0>();
    __syncthreads();
#pragma unroll
    for (int f = 0; f < FR; ++f) read(f, 0, 0);
    auto step = [&](int buf, int kt) {
#pragma unroll
        for (int i = 0; i < TN; ++i) {
#pragma unroll
            for (int f = i * FPR; f < (i + 1) * FPR && f < FR; ++f) read(f, buf, 1);
            __builtin_amdgcn_sched_barrier(0);
            multiply(i, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (kt + NBUF <= steps) wait_requests<(NBUF - 2) * LPS>();
        else wait_requests<0>();
        __syncthreads();
        const bool more = kt + NBUF < steps, next = kt + 1 < steps;
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            if (next) {
#pragma unroll
                for (int f = i * FPR; f < (i + 1) * FPR && f < FR; ++f) read(f, (buf + 1) % NBUF, 0);
            }
            if (more) {
#pragma unroll
                for (int u = i * RPR; u < (i + 1) * RPR && u < LPS; ++u) request(u, kt + NBUF, buf);
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply(i, 1);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    for (int kt = 0; kt < steps; kt += NBUF) {
#pragma unroll
        for (int u = 0; u < NBUF; ++u)
            if (kt + u < steps) step(u, kt + u);
    }

    // NV accumulator tiles make 16 bytes of a token's outputs
    constexpr int NV = OUT == Elem::f32 ? 1 : 2;
    const int n0 = col0 + wn * (BN / WAVES_N) + fq * 4 * NV, m0 = row0 + wm * (BM / WAVES_M) + fr;
    const bool whole = row0 + BM <= p.M && col0 + BN <= p.N;
    f32x4 sw[TN], bias[TN];
    float sx[TM];
#pragma unroll
    for (int i = 0; i < TN; ++i) {
        const int n = n0 + (i / NV) * 16 * NV + (i % NV) * 4;
        sw[i] = four_of(p.step_w, n, p.N);
        bias[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (p.bias) bias[i] = four_of(p.bias, n, p.N);
    }
#pragma unroll
    for (int j = 0; j < TM; ++j) sx[j] = p.step_x[m0 + j * 16 < p.M ? m0 + j * 16 : p.M - 1];
    auto emit = [&](auto inside, auto with_bias) {
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            const int m = m0 + j * 16;
            elem_t<OUT>* y = static_cast<elem_t<OUT>*>(p.Y) + (int64_t)m * p.ldy + n0;
#pragma unroll
            for (int i = 0; i < TN; i += NV) {
                elem_t<OUT> v[4 * NV];
#pragma unroll
                for (int q = 0; q < NV; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float o = (float)acc[i + q][j][e] * (sx[j] * sw[i + q][e]);
                        if constexpr (with_bias.value) o += bias[i + q][e];
                        v[4 * q + e] = float_to_elem<OUT>(o);
                    }
                if (inside.value || (m < p.M && n0 + i * 16 + 4 * NV <= p.N)) {
                    store_piece<OUT>(y + i * 16, v);
                } else if (m < p.M) {
#pragma unroll
                    for (int e = 0; e < 4 * NV; ++e)
                        if (n0 + i * 16 + e < p.N) y[i * 16 + e] = v[e];
                }
            }
        }
    };
    if constexpr (OUT != Elem::f32) {
        // Rows that begin between two words (every second one of an odd pitch): a store of 16 bytes there takes the time of several.  Such a
        // row's lanes store one output further on, with the first of the next lane (the next tiles', behind the last lane), and what that
        // leaves of the wave's columns, the first output and the last, goes by itself (256 x 256 tiles, us without / with: 333 x 2049 x 1052
        // 28.4 / 19.7, 4000 x 6001 x 500 37.0 / 30.8, 8192 x 4097 x 4178 188 / 170; of 4098 outputs 160).
        const bool odd_rows = (((unsigned)(uintptr_t)p.Y >> 1 | (unsigned)p.ldy) & 1) != 0;
        if (odd_rows && col0 + BN <= p.N) {
            constexpr int G = TN / 2;                                  // 16-byte pieces of a lane's outputs of a token
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                const int m = m0 + j * 16;
                unsigned short* y = static_cast<unsigned short*>(p.Y) + (int64_t)m * p.ldy + n0;
                const unsigned odd = ((unsigned)(uintptr_t)y >> 1) & 1;
                unsigned w[G][5];
#pragma unroll
                for (int i = 0; i < TN; ++i)
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        float a = (float)acc[i][j][e] * (sx[j] * sw[i][e]), b = (float)acc[i][j][e + 1] * (sx[j] * sw[i][e + 1]);
                        if (p.bias) {
                            a += bias[i][e];
                            b += bias[i][e + 1];
                        }
                        w[i / 2][i % 2 * 2 + e / 2] = (unsigned)__builtin_bit_cast(unsigned short, float_to_elem<OUT>(a)) |
                                                      (unsigned)__builtin_bit_cast(unsigned short, float_to_elem<OUT>(b)) << 16;
                    }
#pragma unroll
                for (int i = 0; i < G; ++i)                            // (by all lanes, whatever their rows)
                    w[i][4] = (unsigned)__builtin_amdgcn_ds_bpermute(((lane + 16) & 63) * 4, (int)(fq == 0 && i + 1 < G ? w[i + 1 < G ? i + 1 : i][0] : w[i][0]));
                if (m >= p.M) continue;
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    u32x4 r;
#pragma unroll
                    for (int d = 0; d < 4; ++d) r[d] = __builtin_amdgcn_alignbit(w[i][d + 1], w[i][d], odd * 16);
                    unsigned short* to = y + i * 32 + odd;
                    if (i + 1 < G || fq != 3 || odd == 0) {
                        *reinterpret_cast<u32x4_a4*>(to) = r;
                    } else {
                        *reinterpret_cast<u32x2_a4*>(to) = u32x2{r[0], r[1]};
                        *reinterpret_cast<unsigned*>(to + 4) = r[2];
                    }
                }
                if (odd != 0 && (fq == 0 || fq == 3)) {
                    if (fq == 0) y[0] = (unsigned short)w[0][0];
                    else y[(G - 1) * 32 + 7] = (unsigned short)(w[G - 1][3] >> 16);
                }
            }
            return;
        }
    }
    if (whole && p.bias == nullptr) emit(std::true_type{}, std::false_type{});
    else if (whole) emit(std::true_type{}, std::true_type{});
    else emit(std::false_type{}, std::true_type{});
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int NBUF, Elem OUT, bool WIDE = false>
static hipError_t run_rows_tile(RowsGemm p, hipStream_t stream) {
    p.tiles_m = (int)ceil_div(p.M, BM);
    p.tiles_n = (int)ceil_div(p.N, BN);
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n;
    if (total > 0x7FFFFFFF || p.ksteps < 1) return hipErrorInvalidValue;
    return launch_kernel(kTimeGemm, rows_tile_kernel<BM, BN, WAVES_M, WAVES_N, NBUF, OUT, WIDE>, dim3((unsigned)total),
                         dim3(WAVES_M * WAVES_N * 64), 0, stream, p);
}

// Few tiles: 8 XB tokens and 8 WB outputs per workgroup, the steps of K dealt over its NW waves, each with a ring of its own and no
// barrier until the waves' sums meet in LDS.  XB and WB count requests of 8 rows: a matrix tile whose last 8 rows are not there reads
// its first 8 twice.
template <int XB, int WB, int NW, int NBUF, Elem OUT>
__global__ __launch_bounds__(NW * 64) void rows_few_kernel(RowsGemm p) {
    constexpr int XT = (XB + 1) / 2, WT = (WB + 1) / 2, LPS = XB + WB;
    constexpr int STEP = LPS * 1024, RING = NBUF * STEP;
    constexpr int BN = WB * 8, PITCH = BN + 4;              // of the sums: [token][output], 16-byte quads
    static_assert(XB * 8 * PITCH * 4 <= RING, "a wave's sums take its ring's place");
    static_assert(NBUF * LPS < 64, "requests under way");
    extern __shared__ __align__(1024) int8_t rings[];
    const int tid = (int)threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col0 = (int)(blockIdx.x % (unsigned)p.tiles_n) * BN, row0 = (int)(blockIdx.x / (unsigned)p.tiles_n) * (XB * 8);
    const int rows = p.M - row0 < XB * 8 ? p.M - row0 : XB * 8;

    const int piece = (lane & 7) ^ (lane >> 3);
    const int8_t* xbase = p.Xq + (int64_t)row0 * p.ldx;
    const int8_t* wbase = p.Wq + (int64_t)col0 * p.ldw;
    unsigned from[LPS];
#pragma unroll
    for (int u = 0; u < XB; ++u) {
        const int r = u * 8 + (lane >> 3);
        from[u] = (unsigned)((r < rows ? r : rows - 1) * p.ldx + piece * 16);
    }
#pragma unroll
    for (int u = 0; u < WB; ++u) {
        int r = u * 8 + (lane >> 3);
        r = col0 + r < p.N ? r : p.N - 1 - col0;
        from[XB + u] = (unsigned)(r * p.ldw + piece * 16);
    }
    int8_t* ring = rings + wave * RING;
    const unsigned lds0 = lds_address(ring);
    const bool cut = p.ldx < (int64_t)p.ksteps * 128 || p.ldw < (int64_t)p.ksteps * 128;
    const int trips = (p.ksteps - wave + NW - 1) / NW;
    auto fetch = [&](int it, int buf) {
        const int kt = it * NW + wave;
        const int64_t k = (int64_t)kt * 128;
#pragma unroll
        for (int u = 0; u < LPS; ++u) {
            const int8_t* base = (u < XB ? xbase : wbase) + k;
            const unsigned to = lds0 + (unsigned)(buf * STEP + u * 1024);
            if (cut && kt == p.ksteps - 1)
                request_1k(k + piece * 16 < (u < XB ? p.ldx : p.ldw) ? base + from[u] : rows_zero_chunk, to);
            else
                request_1k(base, from[u], to);
        }
    };

    i32x4 acc[WT][XT];
#pragma unroll
    for (int i = 0; i < WT; ++i)
#pragma unroll
        for (int j = 0; j < XT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    const int fr = lane & 15, fq = lane >> 4;
#pragma unroll
    for (int u = 0; u < NBUF; ++u)
        if (u < trips) fetch(u, u);
    for (int it0 = 0; it0 < trips; it0 += NBUF) {
#pragma unroll
        for (int u = 0; u < NBUF; ++u) {
            const int it = it0 + u, left = trips - 1 - it;      // this wave's steps after this one
            if (left < 0) break;
            if (left >= NBUF - 1) wait_requests<(NBUF - 1) * LPS>();
            else if (NBUF > 3 && left == 2) wait_requests<(NBUF > 3 ? 2 : 0) * LPS>();
            else if (NBUF > 2 && left == 1) wait_requests<(NBUF > 2 ? 1 : 0) * LPS>();
            else wait_requests<0>();
            const int8_t* at = ring + u * STEP;
            i32x4 x[2][XT], w[2][WT];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const int slot = ((ks * 4 + fq) ^ (fr & 7)) * 16;
#pragma unroll
                for (int j = 0; j < XT; ++j)
                    x[ks][j] = *reinterpret_cast<const i32x4*>(at + (j * 16 + (2 * j + 1 < XB ? fr : fr & 7)) * 128 + slot);
#pragma unroll
                for (int i = 0; i < WT; ++i)
                    w[ks][i] = *reinterpret_cast<const i32x4*>(at + XB * 1024 + (i * 16 + (2 * i + 1 < WB ? fr : fr & 7)) * 128 + slot);
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int i = 0; i < WT; ++i)
#pragma unroll
                    for (int j = 0; j < XT; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[ks][i], x[ks][j], acc[i][j], 0, 0, 0);
            if (left >= NBUF) {
                __builtin_amdgcn_sched_barrier(0);              // the reads of this buffer have returned: the products took them
                __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
                fetch(it + NBUF, u);
            }
        }
    }
    // every request has landed and every read has returned: the sums take the ring's place
    int32_t* mine = reinterpret_cast<int32_t*>(ring);
#pragma unroll
    for (int i = 0; i < WT; ++i)
#pragma unroll
        for (int j = 0; j < XT; ++j) {
            const int t = j * 16 + fr, n = i * 16 + fq * 4;
            if (t < XB * 8 && n < BN) *reinterpret_cast<i32x4*>(mine + t * PITCH + n) = acc[i][j];
        }
    __syncthreads();
    const int32_t* sums = reinterpret_cast<const int32_t*>(rings);
    for (int o = tid; o < rows * BN; o += NW * 64) {
        const int t = o / BN, c = o - t * BN, m = row0 + t, n = col0 + c;
        if (n >= p.N) continue;
        int a = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) a += sums[w * (RING / 4) + t * PITCH + c];
        float v = (float)a * (p.step_x[m] * p.step_w[n]);
        if (p.bias) v += p.bias[n];
        static_cast<elem_t<OUT>*>(p.Y)[(int64_t)m * p.ldy + n] = float_to_elem<OUT>(v);
    }
}

template <int XB, int WB, int NW, int NBUF, Elem OUT>
static hipError_t run_rows_few(RowsGemm p, hipStream_t stream) {
    constexpr int LDS = NW * NBUF * (XB + WB) * 1024;
    static_assert(LDS <= kMostLds, "a compute unit's LDS");
    p.tiles_m = (int)ceil_div(p.M, XB * 8);
    p.tiles_n = (int)ceil_div(p.N, WB * 8);
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n;
    if (total > 0x7FFFFFFF || p.ksteps < 1) return hipErrorInvalidValue;
    if constexpr (LDS > 65536) {
        static std::atomic<bool> allowed[kMaxDevices];
        const hipError_t e = allow_lds(reinterpret_cast<const void*>(&rows_few_kernel<XB, WB, NW, NBUF, OUT>), LDS, allowed);
        if (e != hipSuccess) return e;
    }
    return launch_kernel(kTimeGemm, rows_few_kernel<XB, WB, NW, NBUF, OUT>, dim3((unsigned)total), dim3(NW * 64),
                         (unsigned)LDS, stream, p);
}

// The layer of few tokens as one launch, codes included.  Every workgroup puts all rows of X on their grids while the first weights are
// on their way (64 pieces of a row at a time per wave, through LDS between the row's maximum and its codes), keeps the codes in LDS as
// images of 8 rows x 128 bytes, and the workgroups share the writing of codes and steps to memory.  Then it goes over its shares of 8 WB
// outputs, its 8 waves with K dealt over them: the weights' requests run two steps ahead of their use, from one share into the next, and
// the waves' sums of a share meet in LDS (integer adds: any order gives the same bits).
// What it buys is the second launch, which costs the host more than the work of a few tokens takes (see launch_forward_rows).
constexpr int kImageWaves = 8, kImageRing = 2, kImageScales = 4, kImageTable = 2048;

// Byte of the image that holds column k of row r.
__device__ __forceinline__ int image_at(int r, int k, int ksteps) {
    return ((r >> 3) * ksteps + (k >> 7)) * 1024 + (r & 7) * 128 + ((((k >> 4) & 7) ^ (r & 7)) << 4) + (k & 15);
}

struct ImageLds {
    int scales, raw, image, sums, rows, table, total;     // byte offsets behind the ring
};
template <int XB, int WB>
__host__ __device__ inline ImageLds image_lds(int segments, int ksteps, int copies) {
    ImageLds l;
    l.scales = kImageWaves * kImageRing * WB * 1024;
    l.raw = l.scales + kImageScales * 256;
    l.image = l.raw + segments * 1024;
    l.sums = l.image + XB * 1024 * ksteps;
    l.rows = l.sums + 2 * XB * 8 * (WB * 8 + 4) * 4;
    l.table = l.rows + 3 * XB * 8 * 4;
    l.total = l.table + (copies * 2 + 15) / 16 * 16;
    return l;
}

// The rows of X into the image, by the whole workgroup; sx: their steps.  Ends with a barrier.
template <Elem T>
__device__ __forceinline__ void quantize_rows(const RowGrids& g, int ksteps, u32x4* raw, int8_t* image, float* sx, float* inv,
                                              unsigned* big, unsigned short* table, int wave, int lane) {
    constexpr int VEC = kVec<T>, NT = kImageWaves * 64, AHEAD = 4;
    const int K = g.C * g.g, Ke = (g.C + g.s) * g.g, pieces = K / VEC, rest = K % VEC, M = (int)g.M, tid = wave * 64 + lane;
    const int per_row = (pieces + (rest ? 1 : 0) + 63) / 64, segments = M * per_row, ldq = (int)g.ldq;
    const auto mine = [&](int r) { return r % (int)gridDim.x == (int)blockIdx.x; };   // rows that this workgroup writes to memory
    if (tid < M) big[tid] = 0u;
    for (int k = K + tid; k < Ke; k += NT) {
        int channel;
        table[k - K] = (unsigned short)source_column(g, k, &channel);
    }
    __syncthreads();
    for (int s0 = wave; s0 < segments; s0 += kImageWaves * AHEAD) {
        u32x4 v[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int s = s0 + a * kImageWaves;
            v[a] = u32x4{0u, 0u, 0u, 0u};
            if (s < segments) {
                const int r = s / per_row, i = (s - r * per_row) * 64 + lane;
                const elem_t<T>* x = static_cast<const elem_t<T>*>(g.X) + (int64_t)r * g.ldx;
                if (i < pieces) v[a] = load_piece<T>(x + i * VEC);
                else if (i == pieces && rest) v[a] = load_partial<T>(x + i * VEC, rest);
            }
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int s = s0 + a * kImageWaves;
            if (s < segments) {
                raw[s * 64 + lane] = v[a];
                unsigned m = 0;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const unsigned q = magnitude(piece_elem<T>(v[a], e));
                    m = q > m ? q : m;
                }
                m = wave_umax32(m);
                if (lane == 0) atomicMax(&big[s / per_row], m);
            }
        }
    }
    __syncthreads();
    if (tid < M) {
        const float thr = g.clip * __uint_as_float(big[tid]), step = __fdiv_rn(thr, g.qmax);
        inv[tid] = inv_step_of(thr, g.qmax);
        sx[tid] = step;
        if (mine(tid)) g.step[tid] = step;
    }
    __syncthreads();
    for (int s = wave; s < segments; s += kImageWaves) {           // (the segments that this wave stored)
        const int r = s / per_row, i = (s - r * per_row) * 64 + lane;
        if (i >= pieces + (rest ? 1 : 0)) continue;
        const u32x4 v = raw[s * 64 + lane];
        const float f = inv[r];
#pragma unroll
        for (int d = 0; d < VEC / 4; ++d) {
            const unsigned code = pack4(code_bits(piece_elem<T>(v, 4 * d), f, g.qmax), code_bits(piece_elem<T>(v, 4 * d + 1), f, g.qmax),
                                        code_bits(piece_elem<T>(v, 4 * d + 2), f, g.qmax), code_bits(piece_elem<T>(v, 4 * d + 3), f, g.qmax));
            *reinterpret_cast<unsigned*>(image + image_at(r, i * VEC + 4 * d, ksteps)) = code;
            if (mine(r) && i < pieces) *reinterpret_cast<unsigned*>(g.Xq + r * g.ldq + i * VEC + 4 * d) = code;
        }
    }
    __syncthreads();
    // left-over columns, copies and padding, from the codes in the image (a word's own left-over bytes are written back as they are)
    const int tail0 = pieces * VEC, end = ldq > ksteps * 128 ? ldq : ksteps * 128, words = (end - tail0) / 4;
    for (int o = tid; o < M * words; o += NT) {
        const int r = o / words, k0 = tail0 + 4 * (o - r * words);
        unsigned word = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int k = k0 + b;
            if (k < Ke) word |= (unsigned)(unsigned char)image[image_at(r, k < K ? k : table[k - K], ksteps)] << (8 * b);
        }
        if (k0 < ksteps * 128) *reinterpret_cast<unsigned*>(image + image_at(r, k0, ksteps)) = word;
        if (mine(r) && k0 < ldq) *reinterpret_cast<unsigned*>(g.Xq + r * g.ldq + k0) = word;
    }
    __syncthreads();
}

template <int XB, int WB, Elem OUT>
__global__ __launch_bounds__(kImageWaves * 64) void rows_image_kernel(RowsGemm p, RowGrids g, int type, int segments) {
    constexpr int NW = kImageWaves, NT = NW * 64, XT = (XB + 1) / 2, WT = (WB + 1) / 2;
    constexpr int STEP = WB * 1024, BN = WB * 8, PITCH = BN + 4, SUMS = XB * 8 * PITCH;
    static_assert(BN <= 32, "the scales of a share are half of a request of 64 words");
    extern __shared__ __align__(1024) int8_t rings[];
    const int tid = (int)threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int8_t* ring = rings + wave * (kImageRing * STEP);
    // the scales of the shares, four in turn (the first wave may ask for those of the share after next while this one's are in use):
    // 32 of step_w, 32 of the bias
    const ImageLds l = image_lds<XB, WB>(segments, p.ksteps, g.s * g.g);
    int8_t* scales = rings + l.scales;
    int8_t* image = rings + l.image;
    int32_t* sums = reinterpret_cast<int32_t*>(rings + l.sums);
    float* sx = reinterpret_cast<float*>(rings + l.rows);
    const unsigned ring0 = lds_address(ring), scales0 = lds_address(scales);

    const int piece = (lane & 7) ^ (lane >> 3);
    const bool cut = p.ldw < (int64_t)p.ksteps * 128;
    const int trips = (p.ksteps - wave + NW - 1) / NW;
    const int shares = (p.tiles_n - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
    // step `it` of this workgroup's share n; with a share's first step go its scales, in the first wave
    auto fetch = [&](int n, int it, int buf) {
        const int col0 = ((int)blockIdx.x + n * (int)gridDim.x) * BN, kt = it * NW + wave;
        const int64_t k = (int64_t)kt * 128;
        if (it == 0 && wave == 0) {
            int c = col0 + (lane & 31);
            c = c < p.N ? c : p.N - 1;
            request_256(lane < 32 || p.bias == nullptr ? p.step_w + c : p.bias + c, scales0 + (unsigned)(n % kImageScales * 256));
        }
        const int8_t* base = p.Wq + (int64_t)col0 * p.ldw + k;
#pragma unroll
        for (int u = 0; u < WB; ++u) {
            int r = u * 8 + (lane >> 3);
            r = col0 + r < p.N ? r : p.N - 1 - col0;
            const unsigned from = (unsigned)(r * p.ldw + piece * 16), to = ring0 + (unsigned)(buf * STEP + u * 1024);
            if (cut && kt == p.ksteps - 1) request_1k(k + piece * 16 < p.ldw ? base + from : rows_zero_chunk, to);
            else request_1k(base, from, to);
        }
    };
    const int total = trips > 0 ? shares * trips : 0;
    int next_n = 0, next_it = 0;                                   // what is to be requested next
    auto fetch_next = [&](int buf) {
        fetch(next_n, next_it, buf);
        if (++next_it == trips) {
            next_it = 0;
            ++next_n;
        }
    };
    if (0 < total) fetch_next(0);
    if (1 < total) fetch_next(1);
    {
        u32x4* raw = reinterpret_cast<u32x4*>(rings + l.raw);
        float* inv = sx + XB * 8;
        unsigned* big = reinterpret_cast<unsigned*>(sx + 2 * XB * 8);
        unsigned short* table = reinterpret_cast<unsigned short*>(rings + l.table);
        if (type == (int)Elem::f32) quantize_rows<Elem::f32>(g, p.ksteps, raw, image, sx, inv, big, table, wave, lane);
        else if (type == (int)Elem::bf16) quantize_rows<Elem::bf16>(g, p.ksteps, raw, image, sx, inv, big, table, wave, lane);
        else quantize_rows<Elem::f16>(g, p.ksteps, raw, image, sx, inv, big, table, wave, lane);
    }
    for (int i = tid; i < 2 * SUMS; i += NT) sums[i] = 0;
    __syncthreads();

    const int fr = lane & 15, fq = lane >> 4;
    int done = 0;
    for (int n = 0; n < shares; ++n) {
        i32x4 acc[WT][XT];
#pragma unroll
        for (int i = 0; i < WT; ++i)
#pragma unroll
            for (int j = 0; j < XT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
        for (int it = 0; it < trips; ++it, ++done) {
            // what may still be under way: the step after this one, with its scales if it begins a share
            if (done + 1 >= total) wait_requests<0>();
            else if (it + 1 == trips && wave == 0) wait_requests<WB + 1>();
            else wait_requests<WB>();
            const int buf = done & 1;
            const int8_t* at = ring + buf * STEP;
            const int8_t* xat = image + (it * NW + wave) * 1024;
            i32x4 x[2][XT], w[2][WT];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const int slot = ((ks * 4 + fq) ^ (fr & 7)) * 16;
#pragma unroll
                for (int j = 0; j < XT; ++j) {                     // (a tile without its last 8 rows reads its first ones twice)
                    const int xb = 2 * j + (2 * j + 1 < XB ? fr >> 3 : 0);
                    x[ks][j] = *reinterpret_cast<const i32x4*>(xat + xb * p.ksteps * 1024 + (fr & 7) * 128 + slot);
                }
#pragma unroll
                for (int i = 0; i < WT; ++i)
                    w[ks][i] = *reinterpret_cast<const i32x4*>(at + (i * 16 + (2 * i + 1 < WB ? fr : fr & 7)) * 128 + slot);
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int i = 0; i < WT; ++i)
#pragma unroll
                    for (int j = 0; j < XT; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[ks][i], x[ks][j], acc[i][j], 0, 0, 0);
            if (done + 2 < total) {
                __builtin_amdgcn_sched_barrier(0);                 // the reads of this buffer have returned: the products took them
                __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
                fetch_next(buf);
            }
        }
        int32_t* meet = sums + (n & 1) * SUMS;
#pragma unroll
        for (int i = 0; i < WT; ++i)
#pragma unroll
            for (int j = 0; j < XT; ++j) {
                const int t = j * 16 + fr, c = i * 16 + fq * 4;
                if (trips > 0 && t < XB * 8 && c < BN) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) atomicAdd(meet + t * PITCH + c + e, acc[i][j][e]);
                }
            }
        // one barrier a share: who reads and clears this share's sums has done so before it comes to the next one's barrier, and the share
        // after that is the next to add to them
        __syncthreads();
        const int col0 = ((int)blockIdx.x + n * (int)gridDim.x) * BN;
        const float* sw = reinterpret_cast<const float*>(scales + n % kImageScales * 256);
        for (int o = tid; o < p.M * BN; o += NT) {
            const int t = o / BN, c = o - t * BN;
            const int a = meet[t * PITCH + c];
            meet[t * PITCH + c] = 0;
            if (col0 + c >= p.N) continue;
            float v = (float)a * (sx[t] * sw[c]);
            if (p.bias) v += sw[32 + c];
            static_cast<elem_t<OUT>*>(p.Y)[(int64_t)t * p.ldy + col0 + c] = float_to_elem<OUT>(v);
        }
    }
}

template <int XB, int WB, Elem OUT>
static hipError_t run_rows_image(RowsGemm p, const RowGrids& g, int type, int segments, hipStream_t stream) {
    const int lds = image_lds<XB, WB>(segments, p.ksteps, g.s * g.g).total;
    if (lds > kMostLds || p.M > XB * 8 || p.ksteps < 1) return hipErrorInvalidValue;
    static std::atomic<bool> allowed[kMaxDevices];
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(&rows_image_kernel<XB, WB, OUT>), kMostLds, allowed);
    if (e != hipSuccess) return e;
    // as many shares for every workgroup as for the busiest
    p.tiles_n = (int)ceil_div(p.N, WB * 8);
    const int64_t rounds = ceil_div(p.tiles_n, compute_units());
    return launch_kernel(kTimeGemm, rows_image_kernel<XB, WB, OUT>, dim3((unsigned)ceil_div(p.tiles_n, rounds)),
                         dim3(kImageWaves * 64), (unsigned)lds, stream, p, g, type, segments);
}

// The kernel by shape.
//
// Up to 32 tokens: the weights' bytes are what is to be had, and every workgroup takes all tokens and a share of the outputs; the
// share grows with the outputs per compute unit, as far as two workgroups' rings fit one (us, one launch after the other: 1 x 6000 x
// 3150 8 / 16 / 24 outputs a workgroup 5.8 / 5.1 / 4.9, 1 x 33001 x 1575 16.3 / 10.8 / 10.9; 20 x 6000 x 3150 8.4 / 7.1 / 5.4, 48 outputs
// of 4 waves 6.5; 20 x 33001 x 1575 33 / 20 / 17, 48 outputs 12.5).
// Beyond, while 64 x 16 (64 x 32) tiles are no more than the compute units, K is dealt over a workgroup's waves all the same (100 x 500 x
// 3150 5.0 against 11.1 in 64 x 64 tiles, 1000 x 256 x 2000 5.6 / 7.9, 300 x 500 x 5000 7.9 / 15.7; 64 x 6000 x 3150 8.6 / 11.0).
// Then tiles: rounds of the chip times what a tile takes, a constant and a cost per step in 10 ns, fitted to tiles of every size alone
// and under load.  128 x 128 comes twice: a ring of three steps, and where there are more tiles than compute units one of two, of which a
// unit holds two workgroups whose ends and starts hide behind each other.  It finds the fastest of the six on these (us, from a graph,
// three sets of operands in turn, 64 x 64 / 128 x 128 / 192 x 128 / 256 x 128 / 256 x 256 / two to a unit):
//   333 x 2049 x 1052 fp16      6.6 /   8.6 /  10.9 /  12.9 /  19.9 /   8.6
//   400 x 8000 x 3150 fp32     25.6 /  19.5 /  24.1 /  28.5 /  43.1 /  22.7
//   700 x 6000 x 3150 fp32     31.7 /  31.8 /  23.3 /  27.9 /  41.5 /  28.1
//   8192 x 4096 x 4178 bf16     227 /   180 /   160 /   145 /   118 /   155
//   700 x 33001 x 1575 fp32     104 /  81.4 /  81.2 /  74.6 /  68.8 /  73.7
//   300 x 33001 x 1575 fp32    49.4 /  41.1 /  43.4 /  51.9 /  53.2 /  39.3
// It knows nothing of the outputs' bytes: the model's 51 us for 700 x 33001 x 1575 are 69.
template <Elem OUT>
static hipError_t run_rows_gemm(const RowsGemm& p, hipStream_t stream) {
    if (p.ldx >= kWidePitch || p.ldw >= kWidePitch) return run_rows_tile<64, 64, 2, 2, 4, OUT, true>(p, stream);
    const int64_t cus = compute_units(), per_cu = ceil_div(ceil_div(p.N, 8), cus);   // requests of 8 outputs a compute unit
#define OCS_ROWS_FEW(XB)                                                        \
    (per_cu <= 2   ? run_rows_few<XB, 2, 8, 2, OUT>(p, stream)                  \
     : per_cu <= 3 ? run_rows_few<XB, 3, 8, 2, OUT>(p, stream)                  \
                   : run_rows_few<XB, XB == 1 ? 4 : 6, XB == 1 ? 8 : 4, 2, OUT>(p, stream))
    if (p.M <= 8) return OCS_ROWS_FEW(1);
    if (p.M <= 16) return OCS_ROWS_FEW(2);
    if (p.M <= 24) return OCS_ROWS_FEW(3);
    if (p.M <= 32) return OCS_ROWS_FEW(4);
#undef OCS_ROWS_FEW
    const int64_t m64 = ceil_div(p.M, 64);
    if (m64 * ceil_div(p.N, 16) <= cus) return run_rows_few<8, 2, 8, 2, OUT>(p, stream);
    if (m64 * ceil_div(p.N, 32) <= cus) return run_rows_few<8, 4, 4, 2, OUT>(p, stream);
    const auto cost = [&](int64_t bm, int64_t bn, int64_t fixed, int64_t step) {
        return ceil_div(ceil_div(p.M, bm) * ceil_div(p.N, bn), cus) * (fixed + step * p.ksteps);
    };
    const int64_t by_tile[6] = {cost(64, 64, 50, 26),    cost(128, 128, 150, 58),  cost(192, 128, 250, 72),
                                cost(256, 128, 350, 92), cost(256, 256, 600, 150),
                                ceil_div(ceil_div(p.M, 128) * ceil_div(p.N, 128), 2 * cus) * (450 + 95 * (int64_t)p.ksteps)};
    int best = 0;
    for (int i = 1; i < 6; ++i)
        if (by_tile[i] < by_tile[best]) best = i;
    switch (best) {
        case 0: return run_rows_tile<64, 64, 2, 2, 4, OUT>(p, stream);
        case 1: return run_rows_tile<128, 128, 2, 4, 3, OUT>(p, stream);
        case 2: return run_rows_tile<192, 128, 2, 4, 3, OUT>(p, stream);
        case 3: return run_rows_tile<256, 128, 4, 2, 3, OUT>(p, stream);
        case 4: return run_rows_tile<256, 256, 2, 4, 2, OUT>(p, stream);
        default: return run_rows_tile<128, 128, 2, 4, 2, OUT>(p, stream);
    }
}

// The layer as one launch where that serves (up to 16 tokens whose rows, codes and rings fit LDS) and pays.  Every workgroup repeats the
// pass over the rows, some 2 us and 0.07 us for each segment of 64 pieces; a launch of its own takes the pass 2.7 us and the host 3.2.
// Outputs that a compute unit has one share of: up to 16 segments where the host launches, up to 8 in a stream that is being captured,
// rows of up to 20 steps (calls one after the other / from a graph, us, two launches and one, weights rotating: 1 x 250 -> 4000 6.9 / 4.7,
// 4.6 / 4.4; 8 x 250 -> 4000, 8 segments, 6.9 / 5.4, 5.0 / 4.8; 4 x 1000 -> 4000, 16, 6.9 / 6.1; 20 x 250 -> 4000, 20, 6.9 / 7.1; 1 x 2000 ->
// 4000 6.9 / 6.0, 6.0 / 5.8; 2 x 3000 -> 4000 7.2 / 7.9).  More shares a unit: not until there are so many that the next share's weights,
// asked for while this one's are summed up, make good for the pass (1 x 1000 -> 12000 6.8 / 7.5; 1 x 500 -> 33001 9.2 / 8.4, 1 x 3000 -> 33001
// 24.6 / 22.7, 4 x 1000 -> 33001, 16 segments, 12.0 / 12.5; rows of two steps 1 x 250 -> 33001 7.7 / 8.1).
template <Elem OUT>
static hipError_t run_forward_rows(const RowsGemm& p, const RowGrids& g, int type, hipStream_t stream, bool* served) {
    *served = false;
    const int64_t K = (int64_t)g.C * g.g, copies = (int64_t)g.s * g.g;
    if (p.M > 16 || copies > kImageTable || p.ldw >= kWidePitch || g.ldq > 65536) return hipSuccess;
    const int64_t segments = p.M * ceil_div(ceil_div(K, type == (int)Elem::f32 ? 4 : 8), 64), cus = compute_units();
    const bool one_share = p.N <= 32 * cus && p.ksteps <= 20 && segments <= 16;
    const bool many_shares = p.N > 128 * cus && p.ksteps >= 4 && segments <= 12;
    if (!one_share && !many_shares) return hipSuccess;
    if (one_share && segments > 8 && stream != nullptr) {          // (the null stream is never captured)
        hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
        const hipError_t e = hipStreamIsCapturing(stream, &status);
        if (e != hipSuccess) return e;
        if (status != hipStreamCaptureStatusNone) return hipSuccess;
    }
    const bool narrow = ceil_div(p.N, 16) <= compute_units();
#define OCS_ROWS_IMAGE(XB)                                                                                             \
    if (p.M <= XB * 8) {                                                                                               \
        *served = image_lds<XB, 4>((int)segments, p.ksteps, (int)copies).total <= kMostLds;                             \
        if (!*served) return hipSuccess;                                                                               \
        return narrow ? run_rows_image<XB, 2, OUT>(p, g, type, (int)segments, stream)                                  \
                      : run_rows_image<XB, 4, OUT>(p, g, type, (int)segments, stream);                                 \
    }
    OCS_ROWS_IMAGE(1)
    OCS_ROWS_IMAGE(2)
#undef OCS_ROWS_IMAGE
    return hipSuccess;
}

// Outputs by the launch: as a rule all of them.  2^28 rows, 2^26 columns and 2^35 outputs are at most 2^23 + 2^22 + 2^20 + 1 tiles of 64 x 64 on 256
// lanes, 2^22 + 2^19 + 1 of 128 x 128 on 512, or 2^21 shares of 32 outputs on 512 where there are few tokens: fewer than kMostLanes.
template <Elem OUT>
static hipError_t run_rows_ranges(const RowsGemm& p, hipStream_t stream) {
    constexpr int64_t kMostRows = (int64_t)1 << 28, kMostColumns = (int64_t)1 << 26, kMostOutputs = (int64_t)1 << 35;
    for (int64_t n0 = 0; n0 < p.N; n0 += kMostColumns) {
        const int64_t cols = p.N - n0 < kMostColumns ? p.N - n0 : kMostColumns;
        const int64_t most = kMostOutputs / cols < kMostRows ? kMostOutputs / cols : kMostRows;
        for (int64_t m0 = 0; m0 < p.M; m0 += most) {
            RowsGemm q = p;
            q.M = (int)(p.M - m0 < most ? p.M - m0 : most);
            q.N = (int)cols;
            q.Xq += m0 * p.ldx;
            q.Wq += n0 * p.ldw;
            q.step_x += m0;
            q.step_w += n0;
            if (p.bias) q.bias += n0;
            q.Y = static_cast<elem_t<OUT>*>(p.Y) + m0 * p.ldy + n0;
            const hipError_t e = run_rows_gemm<OUT>(q, stream);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

hipError_t launch_qgemm_rows(const int8_t* Xq, int64_t ldx, const int8_t* Wq, int64_t ldw, int64_t M, int64_t N, int64_t Kexp,
                             const float* step_x, const float* step_w, const float* bias, void* Y, int out_type, int64_t ldy,
                             hipStream_t stream) {
    const RowsGemm p{Xq, ldx, Wq, ldw, (int)M, (int)N, (int)ceil_div(Kexp, 128), step_x, step_w, bias, Y, ldy, 0, 0};
    switch (static_cast<Elem>(out_type)) {
        case Elem::f32: return run_rows_ranges<Elem::f32>(p, stream);
        case Elem::bf16: return run_rows_ranges<Elem::bf16>(p, stream);
        case Elem::f16: return run_rows_ranges<Elem::f16>(p, stream);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_forward_rows(const void* X, int type, int64_t ldx, int64_t M, int C, int g, int s, const int32_t* chan_src,
                               float clip, float qmax, int8_t* Xq, int64_t ldq, float* step_x, const int8_t* Wq, int64_t ldw,
                               int64_t N, const float* step_w, const float* bias, void* Y, int out_type, int64_t ldy,
                               bool apart, hipStream_t stream) {
    const int64_t Kexp = (int64_t)(C + s) * g;
    const RowsGemm p{Xq, ldq, Wq, ldw, (int)M, (int)N, (int)ceil_div(Kexp, 128), step_x, step_w, bias, Y, ldy, 0, 0};
    const RowGrids rows{X, ldx, M, C, g, s, chan_src, nullptr, clip, qmax, Xq, ldq, step_x};
    if (apart) {                                                   // (one launch reads X and W while outputs are being written)
        bool served = false;
        hipError_t e = hipErrorInvalidValue;
        switch (static_cast<Elem>(out_type)) {
            case Elem::f32: e = run_forward_rows<Elem::f32>(p, rows, type, stream, &served); break;
            case Elem::bf16: e = run_forward_rows<Elem::bf16>(p, rows, type, stream, &served); break;
            case Elem::f16: e = run_forward_rows<Elem::f16>(p, rows, type, stream, &served); break;
        }
        if (e != hipSuccess || served) return e;
    }
    const hipError_t e = launch_row_grids(X, type, ldx, M, C, g, s, chan_src, nullptr, clip, qmax, Xq, ldq, step_x, stream);
    if (e != hipSuccess) return e;
    return launch_qgemm_rows(Xq, ldq, Wq, ldw, M, N, Kexp, step_x, step_w, bias, Y, out_type, ldy, stream);
}

}  // namespace ocs
