// int8 product with a scale per row of either operand: Y[m,n] = acc * (step_x[m] * step_w[n]) + bias[n], acc exact in int32
// on the matrix cores (v_mfma_i32_16x16x64_i8).
//
// The weights are the matrix operand that runs down an accumulator tile and the tokens the one that runs across it: a lane then
// holds four consecutive outputs of one token and stores them as they are, without a detour through LDS.
// Codes go from memory straight into LDS, 128 bytes (one line) of 8 rows per request, 16-byte chunks XOR-ed with the row so that
// the matrix cores' reads of consecutive rows fall into different banks.
#include "row_types.h"

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

// What a row "holds" past its pitch, where that ends inside the last step.
__device__ __align__(16) int8_t rows_zero_chunk[16] = {};

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

// Four outputs of one token, from column n on.
template <Elem OUT>
__device__ __forceinline__ void store4(const RowsGemm& p, int m, int n, i32x4 acc, float sx) {
    if (m >= p.M) return;
    elem_t<OUT>* y = static_cast<elem_t<OUT>*>(p.Y) + (int64_t)m * p.ldy + n;
    elem_t<OUT> v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int c = n + e < p.N ? n + e : p.N - 1;
        float o = (float)acc[e] * (sx * p.step_w[c]);
        if (p.bias) o += p.bias[c];
        v[e] = float_to_elem<OUT>(o);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < p.N) y[e] = v[e];
}

// A BM x BN tile (tokens x outputs) per workgroup, a ring of NBUF steps in LDS.
template <int BM, int BN, int WAVES_M, int WAVES_N, int NBUF, Elem OUT>
__global__ __launch_bounds__(WAVES_M * WAVES_N * 64) void rows_tile_kernel(RowsGemm p) {
    constexpr int NW = WAVES_M * WAVES_N;
    constexpr int XL = BM / 8 / NW, WL = BN / 8 / NW, LPS = XL + WL;
    constexpr int TM = BM / WAVES_M / 16, TN = BN / WAVES_N / 16;
    constexpr int STEP = (BM + BN) * 128;
    static_assert(XL >= 1 && WL >= 1 && BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "whole requests per wave");
    static_assert((NBUF - 1) * LPS < 64 && NBUF >= 2, "requests under way");
    __shared__ __align__(1024) int8_t lds[NBUF * STEP];
    const int tid = (int)threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WAVES_N, wn = wave % WAVES_N;
    const int bm = (int)(blockIdx.x / (unsigned)p.tiles_n), bn = (int)(blockIdx.x % (unsigned)p.tiles_n);
    const int row0 = bm * BM, col0 = bn * BN;

    // request u of a step: rows 8 (u NW + wave) + lane / 8, chunk slot lane % 8 of the step's image
    const int piece = (lane & 7) ^ (lane >> 3);
    const int8_t* xsrc[XL];
    const int8_t* wsrc[WL];
#pragma unroll
    for (int u = 0; u < XL; ++u) {
        const int r = row0 + (u * NW + wave) * 8 + (lane >> 3);
        xsrc[u] = p.Xq + (int64_t)(r < p.M ? r : p.M - 1) * p.ldx + piece * 16;
    }
#pragma unroll
    for (int u = 0; u < WL; ++u) {
        const int r = col0 + (u * NW + wave) * 8 + (lane >> 3);
        wsrc[u] = p.Wq + (int64_t)(r < p.N ? r : p.N - 1) * p.ldw + piece * 16;
    }
    const unsigned lds0 = lds_address(lds) + (unsigned)wave * 1024;
    auto fetch = [&](int kt, int buf) {
        const int64_t k = (int64_t)kt * 128;
        const bool xin = k + piece * 16 < p.ldx, win = k + piece * 16 < p.ldw;
#pragma unroll
        for (int u = 0; u < XL; ++u)
            request_1k(xin ? xsrc[u] + k : rows_zero_chunk, lds0 + (unsigned)(buf * STEP + u * NW * 1024));
#pragma unroll
        for (int u = 0; u < WL; ++u)
            request_1k(win ? wsrc[u] + k : rows_zero_chunk, lds0 + (unsigned)(buf * STEP + BM * 128 + u * NW * 1024));
    };

    i32x4 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    const int fr = lane & 15, fq = lane >> 4;
    i32x4 xf[2][TM], wf[2][TN];
    auto read = [&](int buf, int ks, i32x4 (&x)[TM], i32x4 (&w)[TN]) {
        const int slot = ((ks * 4 + fq) ^ (fr & 7)) * 16;
        const int8_t* xa = lds + buf * STEP + (wm * (BM / WAVES_M) + fr) * 128 + slot;
        const int8_t* wa = lds + buf * STEP + BM * 128 + (wn * (BN / WAVES_N) + fr) * 128 + slot;
#pragma unroll
        for (int j = 0; j < TM; ++j) x[j] = *reinterpret_cast<const i32x4*>(xa + j * 2048);
#pragma unroll
        for (int i = 0; i < TN; ++i) w[i] = *reinterpret_cast<const i32x4*>(wa + i * 2048);
    };
    auto multiply = [&](i32x4 (&x)[TM], i32x4 (&w)[TN]) {
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i], x[j], acc[i][j], 0, 0, 0);
    };

    const int steps = p.ksteps;
#pragma unroll
    for (int u = 0; u < NBUF - 1; ++u)
        if (u < steps) fetch(u, u);
    if (steps >= NBUF - 1) wait_requests<(NBUF - 2) * LPS>();
    else wait_requests<0>();
    __syncthreads();
    read(0, 0, xf[0], wf[0]);
    auto step = [&](int buf, int kt) {
        const bool more = kt + NBUF - 1 < steps;
        if (more) fetch(kt + NBUF - 1, (buf + NBUF - 1) % NBUF);
        read(buf, 1, xf[1], wf[1]);
        __builtin_amdgcn_sched_barrier(0);
        multiply(xf[0], wf[0]);
        __builtin_amdgcn_sched_barrier(0);
        // step kt + 1 has landed for every wave, and every wave has read step kt: its buffer is free
        if (more) wait_requests<(NBUF - 2) * LPS>();
        else wait_requests<0>();
        __syncthreads();
        if (kt + 1 < steps) read((buf + 1) % NBUF, 0, xf[0], wf[0]);
        __builtin_amdgcn_sched_barrier(0);
        multiply(xf[1], wf[1]);
        __builtin_amdgcn_sched_barrier(0);
    };
    for (int kt = 0; kt < steps; kt += NBUF) {
#pragma unroll
        for (int u = 0; u < NBUF; ++u)
            if (kt + u < steps) step(u, kt + u);
    }

#pragma unroll
    for (int j = 0; j < TM; ++j) {
        const int m = row0 + wm * (BM / WAVES_M) + j * 16 + fr;
        const float sx = p.step_x[m < p.M ? m : p.M - 1];
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            const int n = col0 + wn * (BN / WAVES_N) + i * 16 + fq * 4;
            if (n < p.N) store4<OUT>(p, m, n, acc[i][j], sx);
        }
    }
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int NBUF, Elem OUT>
static hipError_t run_rows_tile(RowsGemm p, hipStream_t stream) {
    p.tiles_m = (int)ceil_div(p.M, BM);
    p.tiles_n = (int)ceil_div(p.N, BN);
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n;
    if (total > 0x7FFFFFFF || p.ksteps < 1) return hipErrorInvalidValue;
    return launch_kernel(kTimeGemm, rows_tile_kernel<BM, BN, WAVES_M, WAVES_N, NBUF, OUT>, dim3((unsigned)total),
                         dim3(WAVES_M * WAVES_N * 64), 0, stream, p);
}

template <Elem OUT>
static hipError_t run_rows_gemm(const RowsGemm& p, hipStream_t stream) {
    return run_rows_tile<128, 128, 2, 2, 3, OUT>(p, stream);
}

hipError_t launch_qgemm_rows(const int8_t* Xq, int64_t ldx, const int8_t* Wq, int64_t ldw, int64_t M, int64_t N, int64_t Kexp,
                             const float* step_x, const float* step_w, const float* bias, void* Y, int out_type, int64_t ldy,
                             hipStream_t stream) {
    const RowsGemm p{Xq, ldx, Wq, ldw, (int)M, (int)N, (int)ceil_div(Kexp, 128), step_x, step_w, bias, Y, ldy, 0, 0};
    switch (static_cast<Elem>(out_type)) {
        case Elem::f32: return run_rows_gemm<Elem::f32>(p, stream);
        case Elem::bf16: return run_rows_gemm<Elem::bf16>(p, stream);
        case Elem::f16: return run_rows_gemm<Elem::f16>(p, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace ocs
