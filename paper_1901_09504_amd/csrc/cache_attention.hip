// Attention over a quantized cache: for a query q of position p, over the positions j <= p (and j > p - window) whose pages are there,
//   s_j = scale * q . k_j,   y = sum_j exp(s_j) v_j / sum_j exp(s_j),   lse = log(sum_j exp(s_j));   none: y = 0, lse = -inf.
//
// One pass over the rows with the running maximum and sum of the softmax.  The cache's heads are shared: the G query heads of each and a
// sequence's tokens make the rows of a tile.  Both products run on the matrix cores (v_mfma_f32_16x16x32_bf16) with the cache's side
// down the accumulator: S^T = K Q^T leaves a lane four scores of one query, which are, as they are, its part of P^T in O^T = V^T P^T.
// Codes of 8 bits and of 4 are exact in bf16, and so are the steps: an 8-bit row's step multiplies scores (keys) or weights (values), a
// block's power of two goes into the number itself.  Queries and weights are taken as sums of bf16 numbers, one for bf16 (8 bits), two
// for fp16 (16 bits, where 11 count), three for fp32 (24): scores are as exact as 32-bit sums, and a weight is rounded like the output.
#include <type_traits>

#include "cache.h"

namespace ocs {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct Attention {
    Cache c;
    Sequences s;
    const void* Q;
    int64_t ldq, hdq;
    int Hq, G;                              // query heads, and of them to a head of the cache
    float scale;                            // times log2(e): scores are exponents of 2 here
    int64_t window, most;                   // 0: no window; no position at or beyond `most` is looked at
    void* Y;
    int64_t ldy, hdy;
    float* lse;
    int parts;                              // of a sequence's positions, `chunk` each
    int64_t chunk;
    float* sums;                            // [parts][T * Hq][D] and maxima and sums [parts][T * Hq][2], where there are parts
    float* stats;
};

template <Elem T>
constexpr int kPieces = T == Elem::bf16 ? 1 : T == Elem::f16 ? 2 : 3;      // bf16 numbers that make one of T

__device__ __forceinline__ unsigned bf16_pair(float lo, float hi) {         // of numbers that are bf16 already
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

__device__ __forceinline__ unsigned bf16_rounded(float lo, float hi) {
    const bf16x2 r = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(unsigned, r);
}

// v[0 .. 7] as N sets of bf16 numbers that add up to them
template <int N>
__device__ __forceinline__ void bf16_sums(float (&v)[8], u32x4 (&out)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const unsigned r = bf16_rounded(v[2 * d], v[2 * d + 1]);
            out[n][d] = r;
            v[2 * d] -= __uint_as_float(r << 16);
            v[2 * d + 1] -= __uint_as_float(r & 0xFFFF0000u);
        }
}

__device__ __forceinline__ f32x4 multiply_bf16(u32x4 a, u32x4 b, f32x4 acc) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
#else
    (void)a;
    (void)b;
    return acc;
#endif
}

// two 4-bit codes of byte `at` of a word, times a power of two
template <int AT>
__device__ __forceinline__ unsigned mx_pair(unsigned codes, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, AT));
#else
    (void)codes;
    (void)scale;
    return 0u;
#endif
}

__device__ __forceinline__ float int8_value(unsigned word, int at) { return (float)(int8_t)(word >> (8 * at)); }

__device__ __forceinline__ float over_quarters_max(float v) {
    v = __builtin_fmaxf(v, __shfl_xor(v, 16));
    return __builtin_fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float over_quarters_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// `BYTES` bytes at an address that is a multiple of its largest power of two
template <int BYTES>
__device__ __forceinline__ void load_bytes(const uint8_t* p, unsigned (&w)[(BYTES + 3) / 4]) {
    typedef unsigned short u16_a1 __attribute__((aligned(1)));
    typedef unsigned u32_a1 __attribute__((aligned(1)));
    typedef unsigned u32x2_a1 __attribute__((ext_vector_type(2), aligned(1)));
    typedef unsigned u32x4_a1 __attribute__((ext_vector_type(4), aligned(1)));
    constexpr int WHOLE = BYTES / 4;
#pragma unroll
    for (int i = 0; i < WHOLE / 4; ++i) {
        const u32x4_a1 v = *reinterpret_cast<const u32x4_a1*>(p + 16 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[4 * i + e] = v[e];
    }
    if constexpr (WHOLE % 4 >= 2) {
        const u32x2_a1 v = *reinterpret_cast<const u32x2_a1*>(p + WHOLE / 4 * 16);
        w[WHOLE / 4 * 4] = v[0];
        w[WHOLE / 4 * 4 + 1] = v[1];
    }
    if constexpr (WHOLE % 2 == 1) w[WHOLE - 1] = *reinterpret_cast<const u32_a1*>(p + 4 * (WHOLE - 1));
    if constexpr (BYTES % 4 != 0) {
        unsigned v = 0;
        if constexpr (BYTES % 4 >= 2) v = *reinterpret_cast<const u16_a1*>(p + 4 * WHOLE);
        if constexpr (BYTES % 4 == 1) v = p[4 * WHOLE];
        if constexpr (BYTES % 4 == 3) v |= (unsigned)p[4 * WHOLE + 2] << 16;
        w[WHOLE] = v;
    }
}

// Tiles of ROWS rows (token by token, a token's G heads together): sequence b's begin at cu[b] G / ROWS + b, which leaves each as many as
// it needs.  Answers the tile's sequence, or -1, the tile's first row, the sequence's first token and how many it has.
template <int ROWS>
__device__ __forceinline__ int tile_sequence(const Attention& p, int tile, int* row0, int* first, int* tokens) {
    auto begin = [&](int b) { return (int64_t)clamp_int(p.s.cu[b], 0, p.s.T) * p.G / ROWS + b; };
    const int after = wave_count(p.s.B, [&](int i) { return begin(i) <= tile; });
    if (after == 0) return -1;
    const int b = after - 1, t0 = clamp_int(p.s.cu[b], 0, p.s.T);
    *first = t0;
    *tokens = clamp_int(p.s.cu[b + 1], t0, p.s.T) - t0;
    const int64_t r = (tile - begin(b)) * ROWS;
    if (r >= (int64_t)*tokens * p.G) return -1;
    *row0 = (int)r;
    return b;
}

constexpr int kAttendWaves = 4;

// 16 rows of a sequence and head per workgroup; its waves take 32 positions at a time in turn and meet at the end.  Keys and values go
// from memory to the lanes that multiply them: of a key a lane has D / 4 columns, a quarter; of a value D / 16, and the accumulator's tile t
// holds column (D / 16) m + t in its row m.
template <Elem T, CacheFormat F, int D>
__global__ __launch_bounds__(kAttendWaves * 64) void attend_rows_kernel(Attention p) {
    constexpr int N = kPieces<T>, KS = D / 32, DT = D / 16, ROWS = 16, NW = kAttendWaves;
    constexpr bool MX = F == CacheFormat::mx4;
    constexpr int KB = MX ? D / 8 : D / 4, VB = MX ? D / 32 : D / 16;       // bytes of a lane's part of a key and of a value
    constexpr int ROWB = MX ? D / 2 : D;
    __shared__ float top_of[NW][ROWS], total_of[NW][ROWS];
    __shared__ __align__(16) float out_of[NW / 2][ROWS][D + 4];
    const int lane = (int)threadIdx.x & 63, fr = lane & 15, fq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = blockIdx.y;
    int row0 = 0, t0 = 0, n = 0;
    const int b = __builtin_amdgcn_readfirstlane(tile_sequence<ROWS>(p, (int)blockIdx.x, &row0, &t0, &n));
    if (b < 0) return;
    row0 = __builtin_amdgcn_readfirstlane(row0);
    t0 = __builtin_amdgcn_readfirstlane(t0);
    n = __builtin_amdgcn_readfirstlane(n);
    const int rows = n * p.G - row0 < ROWS ? n * p.G - row0 : ROWS;
    const int64_t start = p.s.starts[b];

    // this lane's query, and the positions that any of the tile sees
    const int row = row0 + (fr < rows ? fr : rows - 1), token = row / p.G, head = h * p.G + row % p.G;
    const int64_t seen = start + token, from = p.window > 0 ? seen - p.window + 1 : 0;
    const int64_t held = p.most < p.c.cols * p.c.P ? p.most : p.c.cols * p.c.P;
    int64_t end = start + (row0 + rows - 1) / p.G + 1, begin = p.window > 0 ? start + row0 / p.G - p.window + 1 : 0;
    end = end < held ? end : held;
    begin = begin > 0 ? begin & ~(int64_t)31 : 0;
    if (p.parts > 1) {
        begin += blockIdx.z * p.chunk;
        end = begin + p.chunk < end ? begin + p.chunk : end;
    }

    u32x4 q[KS][N];
    {
        const elem_t<T>* x = static_cast<const elem_t<T>*>(p.Q) + (int64_t)(t0 + token) * p.ldq + head * p.hdq + fq * (D / 4);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            float v[8];
#pragma unroll
            for (int g = 0; g < 8 / kVec<T>; ++g) {
                const u32x4 piece = load_piece<T>(x + 8 * s + g * kVec<T>);
#pragma unroll
                for (int e = 0; e < kVec<T>; ++e) v[g * kVec<T> + e] = piece_elem<T>(piece, e);
            }
            if (p.c.kdepth) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= cache_doublings(p.c.kdepth[h * D + fq * (D / 4) + 8 * s + e]);
            }
            bf16_sums<N>(v, q[s]);
        }
    }

    struct Block {                                          // of 32 positions, as they are in memory
        unsigned k[2][(KB + 3) / 4], v[8][(VB + 3) / 4];
        float kstep[2][4], vstep[2][4];                     // 8 bits: of this lane's keys and values
        unsigned kscale[2][KS], vscale[8][2];               // 4 bits: the bytes of its blocks
        bool there[2];
    };
    auto load = [&](int64_t j0, Block& x) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int64_t j = j0 + 16 * g;
            int64_t col = j / p.c.P;
            const int at = (int)(j - col * p.c.P);
            int64_t page = -1;
            if (j < held) page = p.c.table[b * p.c.ldt + col];
            x.there[g] = page >= 0 && page < p.c.pages;
            if (!x.there[g]) page = 0;
            const int64_t r = (page * p.c.H + h) * p.c.P + (x.there[g] ? at : 0);       // of the group's first position
            load_bytes<KB>(static_cast<const uint8_t*>(p.c.keys) + (r + fr) * ROWB + fq * KB, x.k[g]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                load_bytes<VB>(static_cast<const uint8_t*>(p.c.values) + (r + 4 * fq + i) * ROWB + fr * VB, x.v[4 * g + i]);
            if constexpr (MX) {
                const uint8_t* ks = static_cast<const uint8_t*>(p.c.kscales) + (r + fr) * (D / 32);
                const uint8_t* vs = static_cast<const uint8_t*>(p.c.vscales) + (r + 4 * fq) * (D / 32);
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    if (s == 0 || (D / 4) % 32 != 0 || s % 4 == 0) x.kscale[g][s] = ks[(fq * (D / 4) + 8 * s) / 32];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x.vscale[4 * g + i][0] = vs[i * (D / 32) + fr * DT / 32];
                    if constexpr (32 % DT != 0) x.vscale[4 * g + i][1] = vs[i * (D / 32) + (fr * DT + DT - 2) / 32];
                }
            } else {
                const f32x4 ks = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.c.kscales) + r + 4 * fq);
                const f32x4 vs = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.c.vscales) + r + 4 * fq);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x.kstep[g][i] = ks[i];
                    x.vstep[g][i] = vs[i];
                }
            }
        }
    };

    f32x4 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float top = -__builtin_inff(), total = 0.0f;            // total: of this lane's positions
    auto use = [&](int64_t j0, const Block& x) {
        float s[8];
        bool sees[8];
        float most = -__builtin_inff();
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                u32x4 k;
                if constexpr (MX) {
                    const unsigned w = x.k[g][st];
                    const float scale = mx_scale_value(x.kscale[g][(D / 4) % 32 != 0 ? st : st / 4 * 4]);
                    k = u32x4{mx_pair<0>(w, scale), mx_pair<1>(w, scale), mx_pair<2>(w, scale), mx_pair<3>(w, scale)};
                } else {
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        const unsigned w = x.k[g][2 * st + d / 2];
                        k[d] = bf16_pair(int8_value(w, 2 * (d & 1)), int8_value(w, 2 * (d & 1) + 1));
                    }
                }
#pragma unroll
                for (int m = N - 1; m >= 0; --m) a = multiply_bf16(k, q[st][m], a);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t j = j0 + 16 * g + 4 * fq + i;
                sees[4 * g + i] = x.there[g] && j <= seen && j >= from && j < end;
                float v = a[i] * p.scale;
                if constexpr (!MX) v = a[i] * (x.kstep[g][i] * p.scale);
                s[4 * g + i] = sees[4 * g + i] ? v : -__builtin_inff();
                most = s[4 * g + i] > most || s[4 * g + i] != s[4 * g + i] ? s[4 * g + i] : most;
            }
        }
        // (a score that is NaN makes the row NaN by its weight; as a maximum it may be lost)
        const float next = __builtin_fmaxf(top, over_quarters_max(most)), base = next == -__builtin_inff() ? 0.0f : next;
        const float shrink = __builtin_amdgcn_exp2f(top - base);
        top = next;
        total *= shrink;
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[i] = __builtin_amdgcn_exp2f(s[i] - base);
            total += w[i];
        }
        bool nan_value[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (MX) {
                // 255: a NaN for those who see it, nothing for the others
                nan_value[i] = x.vscale[i][0] == 255u || (32 % DT != 0 && x.vscale[i][1] == 255u);
                if (nan_value[i] && sees[i]) w[i] = __uint_as_float(0x7FC00000u);
            } else {
                w[i] = sees[i] ? w[i] * x.vstep[i / 4][i % 4] : 0.0f;
            }
        }
        u32x4 pw[N];
        bf16_sums<N>(w, pw);
#pragma unroll
        for (int t = 0; t < DT; t += 2) {                   // two columns of 8 values at a time
            u32x4 v[2];
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                unsigned a, c;                              // of values 2 d and 2 d + 1: columns t and t + 1 either way
                if constexpr (MX) {
                    unsigned pair[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int i = 2 * d + e;
                        unsigned byte = x.vscale[i][0];
                        if constexpr (32 % DT != 0)
                            if ((fr * DT + t) / 32 != fr * DT / 32) byte = x.vscale[i][1];
                        const float scale = mx_scale_value(nan_value[i] ? 0u : byte);
                        const unsigned word = x.v[i][t / 8];
                        pair[e] = t % 8 == 0 ? mx_pair<0>(word, scale) : t % 8 == 2 ? mx_pair<1>(word, scale) : t % 8 == 4 ? mx_pair<2>(word, scale) : mx_pair<3>(word, scale);
                    }
                    a = __builtin_amdgcn_perm(pair[1], pair[0], 0x05040100u);
                    c = __builtin_amdgcn_perm(pair[1], pair[0], 0x07060302u);
                } else {
                    const unsigned w0 = x.v[2 * d][t / 4], w1 = x.v[2 * d + 1][t / 4];
                    a = bf16_pair(int8_value(w0, t % 4), int8_value(w1, t % 4));
                    c = bf16_pair(int8_value(w0, t % 4 + 1), int8_value(w1, t % 4 + 1));
                }
                v[0][d] = a;
                v[1][d] = c;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[t + e][i] *= shrink;
#pragma unroll
                for (int m = N - 1; m >= 0; --m) acc[t + e] = multiply_bf16(v[e], pw[m], acc[t + e]);
            }
        }
    };
    {
        int64_t j = begin + 32 * wave;
        Block now, next;
        if (j < end) load(j, now);
        for (; j < end; j += 32 * NW) {
            if (j + 32 * NW < end) load(j + 32 * NW, next);
            use(j, now);
            now = next;
        }
    }
    total = over_quarters_sum(total);

    // the waves' sums on one maximum, pairwise; the first wave is left with all
    if (fq == 0) {
        top_of[wave][fr] = top;
        total_of[wave][fr] = total;
    }
    __syncthreads();
    float all = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < NW; ++w) all = __builtin_fmaxf(all, top_of[w][fr]);
    const float base = all == -__builtin_inff() ? 0.0f : all;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) sum += total_of[w][fr] * __builtin_amdgcn_exp2f(top_of[w][fr] - base);
    const float shrink = __builtin_amdgcn_exp2f(top - base);
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][i] *= shrink;
#pragma unroll
    for (int half = NW / 2; half > 0; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < DT; ++t) out_of[wave - half][fr][(4 * fq + i) * DT + t] = acc[t][i];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < DT; ++t) acc[t][i] += out_of[wave][fr][(4 * fq + i) * DT + t];
        __syncthreads();
    }
    if (wave != 0 || fr >= rows) return;
    const int64_t out_row = (int64_t)(t0 + token) * p.Hq + head;
    if (p.parts > 1) {
        const int64_t at = blockIdx.z * ((int64_t)p.s.T * p.Hq) + out_row;
        if (fq == 0) {
            p.stats[2 * at] = all;
            p.stats[2 * at + 1] = sum;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < DT; ++t) p.sums[at * D + (4 * fq + i) * DT + t] = acc[t][i];
        return;
    }
    if (p.lse && fq == 0) p.lse[out_row] = sum > 0.0f ? (all + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f : (sum == 0.0f ? -__builtin_inff() : sum);
    elem_t<T>* y = static_cast<elem_t<T>*>(p.Y) + (int64_t)(t0 + token) * p.ldy + head * p.hdy;
    const float part = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            const int d = (4 * fq + i) * DT + t;
            float v = sum == 0.0f ? 0.0f : acc[t][i] * part;
            if (p.c.vdepth) v *= cache_doublings(p.c.vdepth[h * D + d]);
            y[d] = float_to_elem<T>(v);
        }
}

// The parts of a row put together, one workgroup of D lanes per row.
template <Elem T>
__global__ __launch_bounds__(256) void attend_join_kernel(Attention p) {
    const int64_t rows = (int64_t)p.s.T * p.Hq, row = blockIdx.x;
    const int t = (int)(row / p.Hq), head = (int)(row % p.Hq), d = (int)threadIdx.x, D = p.c.D;
    if (sequence_of(p.s, t) < 0 || d >= D) return;
    float all = -__builtin_inff();
    for (int i = 0; i < p.parts; ++i) all = __builtin_fmaxf(all, p.stats[2 * (i * rows + row)]);
    const float base = all == -__builtin_inff() ? 0.0f : all;
    float sum = 0.0f, v = 0.0f;
    for (int i = 0; i < p.parts; ++i) {
        const float part = p.stats[2 * (i * rows + row) + 1], f = __builtin_amdgcn_exp2f(p.stats[2 * (i * rows + row)] - base);
        sum += part * f;
        v += p.sums[(i * rows + row) * D + d] * f;
    }
    v = sum == 0.0f ? 0.0f : v / sum;
    if (p.c.vdepth) v *= cache_doublings(p.c.vdepth[head / p.G * D + d]);
    static_cast<elem_t<T>*>(p.Y)[t * p.ldy + head * p.hdy + d] = float_to_elem<T>(v);
    if (p.lse && d == 0) p.lse[row] = sum > 0.0f ? (all + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f : (sum == 0.0f ? -__builtin_inff() : sum);
}

struct AttentionPlan {
    int64_t tiles;
    int parts;
    int64_t chunk;
};

// Parts of the positions where the tiles alone leave compute units idle.
static AttentionPlan plan_attention(int64_t T, int64_t B, int64_t H, int64_t Hq, int64_t most, int64_t window) {
    const int64_t G = Hq / H, tiles = T * G / 16 + B, range = window > 0 && window + T < most ? window + T : most;
    AttentionPlan a{tiles, 1, 0};
    const int64_t want = ceil_div(8 * (int64_t)compute_units(), tiles * H), can = ceil_div(range, 32 * kAttendWaves * 2);
    int64_t parts = want < can ? want : can;
    if (parts > 1) {
        a.chunk = round_up(ceil_div(range + 31, parts), 32 * kAttendWaves);
        parts = ceil_div(range + 31, a.chunk);
    }
    a.parts = parts > 1 ? (int)parts : 1;
    return a;
}

size_t cache_attention_workspace_bytes(int64_t T, int64_t B, int64_t H, int64_t Hq, int64_t D, int64_t most, int64_t window) {
    const AttentionPlan a = plan_attention(T, B, H, Hq, most, window);
    return a.parts > 1 ? (size_t)a.parts * (size_t)(T * Hq) * (size_t)(D + 2) * 4 : 0;
}

template <Elem T, CacheFormat F, int D>
static hipError_t run_attention(const Attention& p, const AttentionPlan& a, hipStream_t stream) {
    const hipError_t e = launch_kernel(kTimeGemm, attend_rows_kernel<T, F, D>, dim3((unsigned)a.tiles, (unsigned)p.c.H, (unsigned)p.parts),
                                       dim3(kAttendWaves * 64), 0, stream, p);
    if (e != hipSuccess || p.parts == 1) return e;
    return launch_kernel(0, attend_join_kernel<T>, dim3((unsigned)((int64_t)p.s.T * p.Hq)), dim3(256), 0, stream, p);
}

template <Elem T, CacheFormat F>
static hipError_t run_attention_of(const Attention& p, const AttentionPlan& a, hipStream_t stream) {
    switch (p.c.D) {
        case 32: return run_attention<T, F, 32>(p, a, stream);
        case 64: return run_attention<T, F, 64>(p, a, stream);
        case 96: return run_attention<T, F, 96>(p, a, stream);
        case 128: return run_attention<T, F, 128>(p, a, stream);
        case 160: return run_attention<T, F, 160>(p, a, stream);
        case 192: return run_attention<T, F, 192>(p, a, stream);
        case 224: return run_attention<T, F, 224>(p, a, stream);
        case 256: return run_attention<T, F, 256>(p, a, stream);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_cache_attention(const void* Q, int type, int64_t ldq, int64_t hdq, int Hq, const Sequences& s, int64_t most, int format,
                                  const Cache& c, float scale, int64_t window, void* Y, int64_t ldy, int64_t hdy, float* lse,
                                  void* workspace, hipStream_t stream) {
    const AttentionPlan a = plan_attention(s.T, s.B, c.H, Hq, most, window);
    float* sums = static_cast<float*>(workspace);
    Attention p{c, s, Q, ldq, hdq, Hq, Hq / c.H, scale * 1.44269504088896341f, window, most, Y, ldy, hdy, lse, a.parts, a.chunk, sums, nullptr};
    if (a.parts > 1) p.stats = sums + (int64_t)a.parts * s.T * Hq * c.D;
    const bool mx = format == (int)CacheFormat::mx4;
    switch (static_cast<Elem>(type)) {
        case Elem::f32:
            return mx ? run_attention_of<Elem::f32, CacheFormat::mx4>(p, a, stream) : run_attention_of<Elem::f32, CacheFormat::int8>(p, a, stream);
        case Elem::bf16:
            return mx ? run_attention_of<Elem::bf16, CacheFormat::mx4>(p, a, stream) : run_attention_of<Elem::bf16, CacheFormat::int8>(p, a, stream);
        case Elem::f16:
            return mx ? run_attention_of<Elem::f16, CacheFormat::mx4>(p, a, stream) : run_attention_of<Elem::f16, CacheFormat::int8>(p, a, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace ocs
