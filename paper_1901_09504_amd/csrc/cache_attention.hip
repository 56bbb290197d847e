// Attention over a quantized cache: for a query q of position p, over the positions j <= p (and j > p - window) whose pages are there,
//   s_j = scale * q . k_j,   y = sum_j exp(s_j) v_j / sum_j exp(s_j),   lse = log(sum_j exp(s_j));   none: y = 0, lse = -inf.
//
// One pass over the rows with the running maximum and sum of the softmax.  The cache's heads are shared: the G query heads of each and a
// sequence's tokens make the rows of a tile.  Both products run on the matrix cores (v_mfma_f32_16x16x32_bf16) with the cache's side
// down the accumulator: S^T = K Q^T leaves a lane four scores of one query, which are, as they are, its part of P^T in O^T = V^T P^T.
// Codes of 8 bits and of 4 are exact in bf16, and so are the steps: an 8-bit row's step multiplies scores (keys) or weights (values), a
// block's power of two goes into the number itself.  Queries are taken as sums of bf16 numbers, one for bf16 (8 bits), two for fp16 (16 bits,
// where 11 count), three for fp32 (24): scores are as exact as 32-bit sums.  A weight is two of them, off by 2^-16 of itself at most, or three
// for fp32, so that an output is off by its own rounding.  (One for bf16 would be a second rounding of that size: prompts off 64 bits by 0.0023
// of their norm where two leave 0.0017, in 283 us where two take 330; single tokens, which wait for memory, take as long either way.)
#include <type_traits>

#include "cache.h"
#include "tile_requests.h"

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
    int window, held;                       // 0: no window; no position at or beyond `held` is looked at
    unsigned page_magic;                    // 2^32 / P and one more
    void* Y;
    int64_t ldy, hdy;
    float* lse;
    int tiles, parts, chunk;                // tiles of rows; parts of a sequence's positions, `chunk` each
    float* sums;                            // [parts][T * Hq][D] and maxima and sums [parts][T * Hq][2], where there are parts
    float* stats;
};

template <Elem T>
constexpr int kPieces = T == Elem::bf16 ? 1 : T == Elem::f16 ? 2 : 3;      // bf16 numbers that make one of T
template <Elem T>
constexpr int kWeightPieces = T == Elem::f32 ? 3 : 2;                      // and that make a weight of the values

__device__ __forceinline__ unsigned bf16_pair(float lo, float hi) {         // of numbers that are bf16 already
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

__device__ __forceinline__ unsigned bf16_rounded(float lo, float hi) {
    return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
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

// The largest and the sum over the four lanes that hold one query's scores (lanes l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ void exchange_quarters(float v, float* a, float* b, bool far) {
#if defined(__HIP_DEVICE_COMPILE__)
    const unsigned u = __float_as_uint(v);
    const auto r = far ? __builtin_amdgcn_permlane32_swap(u, u, false, false) : __builtin_amdgcn_permlane16_swap(u, u, false, false);
    *a = __uint_as_float(r[0]);
    *b = __uint_as_float(r[1]);
#else
    *a = *b = v;
    (void)far;
#endif
}
__device__ __forceinline__ float over_quarters_max(float v) {
    float a, b;
    exchange_quarters(v, &a, &b, false);
    exchange_quarters(__builtin_fmaxf(a, b), &a, &b, true);
    return __builtin_fmaxf(a, b);
}
__device__ __forceinline__ float over_quarters_sum(float v) {
    float a, b;
    exchange_quarters(v, &a, &b, false);
    exchange_quarters(a + b, &a, &b, true);
    return a + b;
}

// Bits that any of each 16 neighbouring lanes has.
__device__ __forceinline__ unsigned or_of_16(unsigned v) {
    v |= (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x121, 0xF, 0xF, true);     // lanes of a row turned by 1, 2, 4, 8
    v |= (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x122, 0xF, 0xF, true);
    v |= (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x124, 0xF, 0xF, true);
    return v | (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xF, 0xF, true);
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

// A tile of rows (token by token, a token's G heads together): its sequence, or -1, its first row, and the sequence's first token, tokens and
// first position.
struct TileOf {
    int b, row0, first, tokens;
    int start;
};

// Tiles of ROWS rows: sequence b's begin at cu[b] G / ROWS + b, which leaves each as many as it needs.  (T G is below 2^28.)
template <int ROWS>
__device__ __forceinline__ TileOf tile_sequence(const Attention& p, int tile) {
    TileOf t{-1, 0, 0, 0, 0};
    int begin;
    if (p.s.B <= 64) {                                      // all of them at one look
        const int lane = (int)threadIdx.x & 63, i = lane < p.s.B ? lane : p.s.B - 1;
        const int from = p.s.cu[i], to = p.s.cu[i + 1], at = p.s.starts[i];
        const int t0 = clamp_int(from, 0, p.s.T), n = clamp_int(to, t0, p.s.T) - t0, mine = t0 * p.G / ROWS + i;
        const int after = __popcll(__ballot(lane < p.s.B && mine <= tile));
        if (after == 0) return t;
        t.b = after - 1;
        t.first = __builtin_amdgcn_readlane(t0, after - 1);
        t.tokens = __builtin_amdgcn_readlane(n, after - 1);
        t.start = __builtin_amdgcn_readlane(at, after - 1);
        begin = __builtin_amdgcn_readlane(mine, after - 1);
    } else {
        const int after = wave_count(p.s.B, [&](int i) { return clamp_int(p.s.cu[i], 0, p.s.T) * p.G / ROWS + i <= tile; });
        if (after == 0) return t;
        t.b = after - 1;
        t.first = clamp_int(p.s.cu[t.b], 0, p.s.T);
        t.tokens = clamp_int(p.s.cu[t.b + 1], t.first, p.s.T) - t.first;
        t.start = p.s.starts[t.b];
        begin = t.first * p.G / ROWS + t.b;
    }
    t.row0 = (tile - begin) * ROWS;
    if (t.row0 < 0 || t.row0 >= t.tokens * p.G) t.b = -1;       // (below 0 where offsets do not ascend)
    return t;
}

// What a query sees: `count` positions from `from` on (no position beyond kMostPositions is looked at).
struct Seen {
    int from, count;
};
__device__ __forceinline__ Seen positions_seen(const Attention& p, int64_t position) {
    const int64_t last = position < p.held ? position : p.held - 1, first = p.window > 0 && position >= p.window ? position - p.window + 1 : 0;
    Seen s{0, 0};
    if (first <= last) s = Seen{(int)first, (int)(last - first + 1)};
    return s;
}

// The row of the pool (of head 0, counted in [pages, H, P]) where 16 positions from j on begin, or -1.  The page's number comes first: what
// it costs is the look-up in the table, which callers make one block of positions ahead.
struct PageAt {
    int page, at;
};
__device__ __forceinline__ PageAt page_of(const Attention& p, const int32_t* table, int j, int end) {
    int col = (int)__umulhi((unsigned)j, p.page_magic), at = j - col * p.c.P;          // col is j / P or one more
    if (at < 0) {
        col -= 1;
        at += p.c.P;
    }
    return PageAt{j < end ? table[col] : -1, at};
}

// The same for tiles of many rows, those that see most first: what a workgroup takes goes with the positions that its rows see, and one that
// begins last should not be the longest.  A sequence's tiles go backwards; up to 64 sequences go by length.  (Prompts of 512 to 1501 tokens in
// sequences of 1501 to 6001, 8 heads: in the order given 428 us, so 345.)
template <int ROWS>
__device__ __forceinline__ TileOf long_tile_sequence(const Attention& p, int tile) {
    if (p.s.B > 64) {
        TileOf t = tile_sequence<ROWS>(p, tile);
        t.row0 = (t.tokens * p.G + ROWS - 1) / ROWS * ROWS - ROWS - t.row0;
        return t;
    }
    const int lane = (int)threadIdx.x & 63;
    int t0 = 0, n = 0, tiles = 0, before = 0, start = 0;
    if (lane < p.s.B) {
        start = p.s.starts[lane];
        t0 = clamp_int(p.s.cu[lane], 0, p.s.T);
        n = clamp_int(p.s.cu[lane + 1], t0, p.s.T) - t0;
        tiles = (n * p.G + ROWS - 1) / ROWS;
    }
    const int64_t length = (int64_t)start + n;
    const int size = (int)(length < 0 ? 0 : length < 0x7FFFFFFF ? length : 0x7FFFFFFF);
    for (int j = 0; j < p.s.B; ++j) {
        const int other = __builtin_amdgcn_readlane(size, j), more = __builtin_amdgcn_readlane(tiles, j);
        if (other > size || (other == size && j < lane)) before += more;
    }
    const uint64_t which = __ballot(tile >= before && tile < before + tiles);
    TileOf t{-1, 0, 0, 0, 0};
    if (which == 0) return t;
    t.b = __builtin_ctzll(which);
    t.first = __builtin_amdgcn_readlane(t0, t.b);
    t.tokens = __builtin_amdgcn_readlane(n, t.b);
    t.start = __builtin_amdgcn_readlane(start, t.b);
    t.row0 = (__builtin_amdgcn_readlane(before + tiles, t.b) - 1 - tile) * ROWS;
    return t;
}

// How far above the softmax's reference a score may be before the sums are put on a new one (in powers of two): the reference then hardly
// ever changes after the first positions, and weights stay far inside fp32's and bf16's range.
constexpr float kSlack = 8.0f;

// Scale bytes of values from here on are no numbers: 255 by definition, the two below it because 6 times their power of two is beyond
// bf16 (no row that was written has them, but rubbish where nothing is seen may, and infinity times a weight of 0 is NaN).  One such block makes
// the row none, whichever it is.
constexpr unsigned kNoNumber = 253;

// whether any of four scale bytes is no number: their low seven bits carry into the eighth, which is set
__device__ __forceinline__ bool any_no_number(unsigned bytes) {
    return (((bytes & 0x7F7F7F7Fu) + (256 - kNoNumber) * 0x01010101u) & bytes & 0x80808080u) != 0u;
}

constexpr int kAttendWaves = 4;

// The columns of a key that a lane of quarter `fq` multiplies in step s of the product: 8 from here on.  Steps go in groups, for which a
// lane loads up to 16 bytes, 64 of a row between the four quarters; queries take the same order.
template <bool MX, int D>
struct KeyColumns {
    static constexpr int STEPS = D / 32, MOST = MX ? 4 : 2;
    static constexpr int start(int s) { return s / MOST * MOST; }
    static constexpr int steps(int s) { return STEPS - start(s) < MOST ? STEPS - start(s) : MOST; }
    static __device__ __forceinline__ int column(int s, int fq) { return 32 * start(s) + 8 * (steps(s) * fq + s - start(s)); }
};

// A lane's part of a key, a group of steps after the other.
template <bool MX, int D, int S>
__device__ __forceinline__ void load_key(const uint8_t* key, int fq, unsigned* w) {
    if constexpr (S < D / 32) {
        constexpr int BYTES = (MX ? 4 : 8) * KeyColumns<MX, D>::steps(S);
        unsigned part[BYTES / 4];
        load_bytes<BYTES>(key + (MX ? 16 : 32) * S + BYTES * fq, part);
#pragma unroll
        for (int i = 0; i < BYTES / 4; ++i) w[(MX ? 1 : 2) * S + i] = part[i];
        load_key<MX, D, S + KeyColumns<MX, D>::steps(S)>(key, fq, w);
    }
}

// Workgroups are dealt to the 8 XCDs in turn: heads come first among them, so that every XCD gets its share of each sequence (64 sequences
// of 128 to 8192 positions, 8 heads, tiles first 163 us, heads first 147).
//
// 16 rows of a sequence and head per workgroup; its waves take 32 positions at a time in turn and meet at the end.  Keys and values go
// from memory to the lanes that multiply them: of a key a lane has D / 4 columns, of a value D / 16, and the accumulator's tile t
// holds column (D / 16) m + t in its row m.  Bound by the rows' bytes: 64 sequences to 8192 positions, 8 heads of 128 in 8 bits, 128 us, 4.4 TB/s;
// the loads alone, nothing made of them, take 5 us less.
template <Elem T, CacheFormat F, int D>
__global__ __launch_bounds__(kAttendWaves * 64, 2) void attend_rows_kernel(Attention p) {
    constexpr int N = kPieces<T>, NV = kWeightPieces<T>, KS = D / 32, DT = D / 16, ROWS = 16, NW = kAttendWaves;
    constexpr bool MX = F == CacheFormat::mx4;
    constexpr int KB = MX ? D / 8 : D / 4, VB = MX ? D / 32 : D / 16;       // bytes of a lane's part of a key and of a value
    using Columns = KeyColumns<MX, D>;
    constexpr int ROWB = MX ? D / 2 : D;
    __shared__ float top_of[NW][ROWS], total_of[NW][ROWS];
    __shared__ __align__(16) float out_of[NW / 2][ROWS][D + 4];
    const int lane = (int)threadIdx.x & 63, fr = lane & 15, fq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = (int)(blockIdx.x % (unsigned)p.c.H), part = (int)(blockIdx.x / (unsigned)p.c.H / (unsigned)p.tiles);
    const TileOf tile = tile_sequence<ROWS>(p, (int)(blockIdx.x / (unsigned)p.c.H % (unsigned)p.tiles));
    const int b = __builtin_amdgcn_readfirstlane(tile.b);
    if (b < 0) return;
    const int row0 = __builtin_amdgcn_readfirstlane(tile.row0), t0 = __builtin_amdgcn_readfirstlane(tile.first);
    const int n = __builtin_amdgcn_readfirstlane(tile.tokens);
    const int rows = n * p.G - row0 < ROWS ? n * p.G - row0 : ROWS;
    const int64_t start = __builtin_amdgcn_readfirstlane(tile.start);

    // this lane's query, and the positions that any of the tile sees and that all of it see
    const int row = row0 + (fr < rows ? fr : rows - 1), token = row / p.G, head = h * p.G + row % p.G;
    const int first_token = row0 / p.G, last_token = (row0 + rows - 1) / p.G;
    const Seen mine = positions_seen(p, start + token), first = positions_seen(p, start + first_token), last = positions_seen(p, start + last_token);
    const int64_t first_seen = start + first_token - p.window + 1, past = start + last_token + 1;
    int begin = p.window > 0 && first_seen > 0 ? (int)(first_seen < p.held ? first_seen & ~(int64_t)31 : p.held) : 0;
    int end = past < 0 ? 0 : past < p.held ? (int)past : p.held;
    const int all_from = last.count > 0 ? last.from : 0x7FFFFFFF, all_end = first.from + first.count;
    if (p.parts > 1) {
        const int64_t at = begin + part * (int64_t)p.chunk;
        begin = at < end ? (int)at : end;
        end = at + p.chunk < end ? (int)(at + p.chunk) : end;
    }

    u32x4 q[KS][N];
    {
        const elem_t<T>* x = static_cast<const elem_t<T>*>(p.Q) + (int64_t)(t0 + token) * p.ldq + head * p.hdq;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            float v[8];
#pragma unroll
            for (int g = 0; g < 8 / kVec<T>; ++g) {
                const u32x4 piece = load_piece<T>(x + Columns::column(s, fq) + g * kVec<T>);
#pragma unroll
                for (int e = 0; e < kVec<T>; ++e) v[g * kVec<T> + e] = piece_elem<T>(piece, e);
            }
            if (p.c.kdepth) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= cache_doublings(p.c.kdepth[h * D + Columns::column(s, fq) + e]);
            }
            bf16_sums<N>(v, q[s]);
        }
    }

    struct Block {                                          // of 32 positions, as they are in memory
        unsigned k[2][(KB + 3) / 4], v[8][(VB + 3) / 4];
        float kstep[2][4], vstep[2][4];                     // 8 bits: of this lane's keys and values
        unsigned kscale[2][KS], vscale[8][2];               // 4 bits: the bytes of its blocks
    };
    struct Where {                                          // its pages
        PageAt at[2];
    };
    const int32_t* table = p.c.table + b * p.c.ldt;
    auto look_up = [&](int j0, Where& w) {
#pragma unroll
        for (int g = 0; g < 2; ++g) w.at[g] = page_of(p, table, j0 + 16 * g, end);
    };
    auto there = [&](const PageAt& at) { return at.page >= 0 && at.page < p.c.pages; };
    auto first_row = [&](const PageAt& at) {                // of the group's first position
        const bool ok = there(at);
        return ((int64_t)(ok ? at.page : 0) * p.c.H + h) * p.c.P + (ok ? at.at : 0);
    };
    auto load_keys = [&](const Where& w, Block& x) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int64_t r = first_row(w.at[g]);
            load_key<MX, D, 0>(static_cast<const uint8_t*>(p.c.keys) + r * ROWB + fr * ROWB, fq, x.k[g]);
            if constexpr (MX) {
                const uint8_t* ks = static_cast<const uint8_t*>(p.c.kscales) + r * (D / 32) + fr * (D / 32);
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    if (Columns::steps(s) != 4 || s % 4 == 0) x.kscale[g][s] = ks[Columns::column(s, fq) / 32];
            } else {
                const f32x4 ks = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.c.kscales) + r + 4 * fq);
#pragma unroll
                for (int i = 0; i < 4; ++i) x.kstep[g][i] = ks[i];
            }
        }
    };
    auto load_values = [&](const Where& w, Block& x) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int64_t r = first_row(w.at[g]);
            const uint8_t* values = static_cast<const uint8_t*>(p.c.values) + r * ROWB;
#pragma unroll
            for (int i = 0; i < 4; ++i) load_bytes<VB>(values + (4 * fq + i) * ROWB + fr * VB, x.v[4 * g + i]);
            if constexpr (MX) {
                const uint8_t* vs = static_cast<const uint8_t*>(p.c.vscales) + r * (D / 32) + 4 * fq * (D / 32);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x.vscale[4 * g + i][0] = vs[i * (D / 32) + fr * DT / 32];
                    if constexpr (32 % DT != 0) x.vscale[4 * g + i][1] = vs[i * (D / 32) + (fr * DT + DT - 2) / 32];
                }
            } else {
                const f32x4 vs = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.c.vscales) + r + 4 * fq);
#pragma unroll
                for (int i = 0; i < 4; ++i) x.vstep[g][i] = vs[i];
            }
        }
    };

    f32x4 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float top = -__builtin_inff(), total = 0.0f;            // the softmax's reference; the sum over this lane's positions
    // Positions j0 on; the next ones' keys and values (more: there are some) take the place of these as soon as they have been multiplied.
    auto use = [&](int j0, const Where& where, Block& x, bool more, const Where& next) {
        float s[8];
        // whether every row of the tile sees all 32
        const bool whole = j0 >= all_from && j0 + 32 <= all_end && j0 + 32 <= end && there(where.at[0]) && there(where.at[1]);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                u32x4 k;
                if constexpr (MX) {
                    const unsigned w = x.k[g][st];
                    const float scale = mx_scale_value(x.kscale[g][Columns::steps(st) != 4 ? st : st / 4 * 4]);
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
            for (int i = 0; i < 4; ++i) s[4 * g + i] = MX ? a[i] * p.scale : a[i] * (x.kstep[g][i] * p.scale);
        }
        if (more) load_keys(next, x);
        unsigned sees = 0xFFu;                              // a bit per position of this lane
        if (!whole) {
            sees = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int j = j0 + 16 * (i / 4) + 4 * fq + i % 4;
                if (there(where.at[i / 4]) && j < end && (unsigned)(j - mine.from) < (unsigned)mine.count) sees |= 1u << i;
                else s[i] = -__builtin_inff();
            }
        }
        float most = s[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) most = __builtin_fmaxf(most, s[i]);
        if (__any(most > top + kSlack)) {                   // (the lanes of a query take the same reference: they all come here)
            const float next = __builtin_fmaxf(top, over_quarters_max(most));
            const float shrink = next == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(top - next);
            top = next;
            total *= shrink;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[t][i] *= shrink;
        }
        const float base = top == -__builtin_inff() ? 0.0f : top;
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[i] = __builtin_amdgcn_exp2f(s[i] - base);
            total += w[i];
        }
        unsigned vscale[8][2];
        if constexpr (MX) {
            unsigned highest = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < (32 % DT != 0 ? 2 : 1); ++e) {
                    vscale[i][e] = x.vscale[i][e];
                    highest = vscale[i][e] > highest ? vscale[i][e] : highest;
                }
            if (__any(highest >= kNoNumber)) {              // a NaN for those who see it, nothing for the others
                unsigned bad = 0;                           // a bit per position; its blocks are those of the quarter's 16 lanes
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (vscale[i][0] >= kNoNumber || (32 % DT != 0 && vscale[i][1] >= kNoNumber)) {
                        bad |= 1u << i;
                        vscale[i][0] = vscale[i][1] = 127u;
                    }
                bad = or_of_16(bad) & sees;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (bad >> i & 1) w[i] = __uint_as_float(0x7FC00000u);
            }
        } else if (whole) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] *= x.vstep[i / 4][i % 4];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = sees >> i & 1 ? w[i] * x.vstep[i / 4][i % 4] : 0.0f;
        }
        u32x4 pw[NV];
        bf16_sums<NV>(w, pw);
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
                        unsigned byte = vscale[i][0];
                        if constexpr (32 % DT != 0)
                            if ((fr * DT + t) / 32 != fr * DT / 32) byte = vscale[i][1];
                        const float scale = mx_scale_value(byte);
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
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int m = NV - 1; m >= 0; --m) acc[t + e] = multiply_bf16(v[e], pw[m], acc[t + e]);
        }
        if (more) load_values(next, x);
    };
    {
        // pages are looked up two blocks ahead, rows asked for most of a block ahead
        constexpr int STRIDE = 32 * NW;
        int j = begin + 32 * wave;
        Block x;
        Where now{}, next{};
        if (j < end) {
            look_up(j, now);
            look_up(j + STRIDE, next);
            load_keys(now, x);
            load_values(now, x);
        }
        for (; j < end; j += STRIDE) {
            Where further;
            look_up(j + 2 * STRIDE, further);
            use(j, now, x, j + STRIDE < end, next);
            now = next;
            next = further;
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
        const int64_t at = part * ((int64_t)p.s.T * p.Hq) + out_row;
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
    const float share = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            const int d = (4 * fq + i) * DT + t;
            float v = sum == 0.0f ? 0.0f : acc[t][i] * share;
            if (p.c.vdepth) v *= cache_doublings(p.c.vdepth[h * D + d]);
            y[d] = float_to_elem<T>(v);
        }
}

// Of 4 rows of 16 two-byte numbers in LDS, to which 16 lanes give the addresses of 8 bytes each, lane i gets column i.
__device__ __forceinline__ u32x2 read_transposed(const uint8_t* lds) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)lds));
#else
    (void)lds;
    return u32x2{0u, 0u};
#endif
}

// Many rows: 64 NT rows of a sequence and head per workgroup, 16 NT to each of its four waves.  The workgroup turns KT positions at a time into
// bf16 numbers in LDS, once for all its rows, while the next positions' codes are on their way, and the waves multiply from there: keys a
// row at a time, values transposed as they are read (ds_read_b64_tr_b16).  Rows of LDS are 4 and 8 banks apart beyond a multiple of 64, so
// that what the matrix cores read at a time lies in different banks.  Bound by vector instructions (conversions, exponentials, factors, the weights' second halves: 51 % of
// the time) and matrix cores (35 %), which overlap little: prompts of 512 to 1501 tokens in sequences to 6001, 32 heads on 8 of 128, 330 us, 0.57 PFLOP/s
// (4 bits 313; fp16 queries 366, fp32 472).
constexpr int kTileWaves = 4;
template <Elem T, int D>
struct AttendTile {
    static constexpr int N = kPieces<T>;
    static constexpr int THREADS = 64 * kTileWaves;
    static constexpr int NT = D <= 128 ? 2 : 1, ROWS = 16 * kTileWaves * NT, KT = D <= 128 && N == 1 ? 64 : 32;
    static constexpr int KPITCH = 2 * D + 16, VPITCH = 2 * D + 32;
    static constexpr int LDS = 2 * KT * (KPITCH + VPITCH);
};

template <Elem T, CacheFormat F, int D>
__global__ __launch_bounds__(kTileWaves * 64, 8 / kTileWaves) void attend_tile_kernel(Attention p) {
    using Tile = AttendTile<T, D>;
    constexpr int N = Tile::N, NT = Tile::NT, ROWS = Tile::ROWS, KT = Tile::KT, KPITCH = Tile::KPITCH, VPITCH = Tile::VPITCH, THREADS = Tile::THREADS;
    constexpr int NV = kWeightPieces<T>, KS = D / 32, DT = D / 16, MT = KT / 16;
    constexpr bool MX = F == CacheFormat::mx4;
    constexpr int ROWB = MX ? D / 2 : D, PIECE = MX ? 8 : 16;              // bytes of a row, and of 16 of its codes
    constexpr int ITEMS = KT * (D / 16), LOADS = (ITEMS + THREADS - 1) / THREADS;
    extern __shared__ __align__(16) uint8_t lds[];
    __shared__ __align__(16) float ksteps[2][KT], vsteps[2][KT];
    __shared__ int there_of[2][MT];
    const int tid = (int)threadIdx.x, lane = tid & 63, fr = lane & 15, fq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = (int)(blockIdx.x % (unsigned)p.c.H), part = (int)(blockIdx.x / (unsigned)p.c.H / (unsigned)p.tiles);
    const TileOf tile = long_tile_sequence<ROWS>(p, (int)(blockIdx.x / (unsigned)p.c.H % (unsigned)p.tiles));
    const int b = __builtin_amdgcn_readfirstlane(tile.b);
    if (b < 0) return;
    const int row0 = __builtin_amdgcn_readfirstlane(tile.row0), t0 = __builtin_amdgcn_readfirstlane(tile.first);
    const int n = __builtin_amdgcn_readfirstlane(tile.tokens);
    const int rows = n * p.G - row0 < ROWS ? n * p.G - row0 : ROWS;
    const int64_t start = __builtin_amdgcn_readfirstlane(tile.start);
    const int first_token = row0 / p.G, last_token = (row0 + rows - 1) / p.G;
    const Seen first = positions_seen(p, start + first_token), last = positions_seen(p, start + last_token);
    const int64_t first_seen = start + first_token - p.window + 1, past = start + last_token + 1;
    int begin = p.window > 0 && first_seen > 0 ? (int)(first_seen < p.held ? first_seen & ~(int64_t)31 : p.held) : 0;
    int end = past < 0 ? 0 : past < p.held ? (int)past : p.held;
    const int all_from = last.count > 0 ? last.from : 0x7FFFFFFF, all_end = first.from + first.count;
    if (p.parts > 1) {
        const int64_t at = begin + part * (int64_t)p.chunk;
        begin = at < end ? (int)at : end;
        end = at + p.chunk < end ? (int)(at + p.chunk) : end;
    }

    // this lane's queries, and the positions that the wave sees
    const int wave_row = wave * 16 * NT;
    int token[NT], head[NT];
    Seen mine[NT];
    u32x4 q[NT][KS][N];
    int wave_from = 0x7FFFFFFF, wave_end = 0;
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        const int r = wave_row + 16 * u + fr, row = row0 + (r < rows ? r : rows - 1);
        token[u] = row / p.G;
        head[u] = h * p.G + row - token[u] * p.G;
        mine[u] = positions_seen(p, start + token[u]);
        if (r >= rows) mine[u].count = 0;
        const elem_t<T>* x = static_cast<const elem_t<T>*>(p.Q) + (int64_t)(t0 + token[u]) * p.ldq + head[u] * p.hdq + 8 * fq;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            float v[8];
#pragma unroll
            for (int g = 0; g < 8 / kVec<T>; ++g) {
                const u32x4 piece = load_piece<T>(x + 32 * s + g * kVec<T>);
#pragma unroll
                for (int e = 0; e < kVec<T>; ++e) v[g * kVec<T> + e] = piece_elem<T>(piece, e);
            }
            if (p.c.kdepth) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= cache_doublings(p.c.kdepth[h * D + 32 * s + 8 * fq + e]);
            }
            bf16_sums<N>(v, q[u][s]);
        }
    }
    if (wave_row < rows) {
        const int last_row = wave_row + 16 * NT < rows ? wave_row + 16 * NT - 1 : rows - 1;
        const int64_t from = start + (row0 + wave_row) / p.G - p.window + 1, to = start + (row0 + last_row) / p.G + 1;
        wave_from = p.window > 0 && from > 0 ? (int)(from < p.held ? from : p.held) : 0;
        wave_end = to < 0 ? 0 : to < p.held ? (int)to : p.held;
    }

    // codes of KT positions on their way: 16 of a key and of a value to a lane
    struct Codes {
        unsigned k[PIECE / 4], v[PIECE / 4];
        float kstep, vstep;                                 // 4 bits: of the key, the scale byte's number
        unsigned vscale[(D / 32 + 3) / 4];                  // and the value's scale bytes, all of them
    };
    Codes codes[LOADS];
    int page[LOADS], row_of[LOADS];
    bool there[LOADS];
    const int32_t* table = p.c.table + b * p.c.ldt;
    const unsigned pages = (unsigned)p.c.pages, page_rows = (unsigned)p.c.H * (unsigned)p.c.P;
    const uint8_t* const keys = static_cast<const uint8_t*>(p.c.keys) + (int64_t)h * p.c.P * ROWB;
    const uint8_t* const values = static_cast<const uint8_t*>(p.c.values) + (int64_t)h * p.c.P * ROWB;
    const uint8_t* const kscales = static_cast<const uint8_t*>(p.c.kscales) + (int64_t)h * p.c.P * (MX ? D / 32 : 4);
    const uint8_t* const vscales = static_cast<const uint8_t*>(p.c.vscales) + (int64_t)h * p.c.P * (MX ? D / 32 : 4);
    auto key_of = [&](int u) { return (tid + THREADS * u) / (D / 16); };
    auto part_of = [&](int u) { return (tid + THREADS * u) % (D / 16); };
    auto look_up = [&](int j0) {                             // (positions behind the last repeat it)
#pragma unroll
        for (int u = 0; u < LOADS; ++u)
            if (ITEMS % THREADS == 0 || tid + THREADS * u < ITEMS) {
                const int j = j0 + key_of(u) < end ? j0 + key_of(u) : end - 1;
                int col = (int)__umulhi((unsigned)j, p.page_magic), at = j - col * p.c.P;
                col -= at < 0;
                row_of[u] = at < 0 ? at + p.c.P : at;
                page[u] = table[col];
            }
    };
    auto load = [&]() {
#pragma unroll
        for (int u = 0; u < LOADS; ++u)
            if (ITEMS % THREADS == 0 || tid + THREADS * u < ITEMS) {
                there[u] = (unsigned)page[u] < pages;
                const uint64_t r = (uint64_t)(there[u] ? (unsigned)page[u] : 0u) * page_rows + (unsigned)row_of[u];
                load_bytes<PIECE>(keys + r * ROWB + part_of(u) * PIECE, codes[u].k);
                load_bytes<PIECE>(values + r * ROWB + part_of(u) * PIECE, codes[u].v);
                if constexpr (MX) {
                    codes[u].kstep = mx_scale_value(kscales[r * (D / 32) + part_of(u) / 2]);
                    load_bytes<D / 32>(vscales + r * (D / 32), codes[u].vscale);
                } else {
                    codes[u].kstep = *reinterpret_cast<const float*>(kscales + r * 4);
                    codes[u].vstep = *reinterpret_cast<const float*>(vscales + r * 4);
                }
            }
    };
    auto numbers = [&](const unsigned (&w)[PIECE / 4], float step, u32x4 (&out)[2]) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if constexpr (MX) {
                out[e] = u32x4{mx_pair<0>(w[e], step), mx_pair<1>(w[e], step), mx_pair<2>(w[e], step), mx_pair<3>(w[e], step)};
            } else {
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const unsigned c = w[2 * e + d / 2];
                    out[e][d] = bf16_pair(int8_value(c, 2 * (d & 1)), int8_value(c, 2 * (d & 1) + 1));
                }
            }
    };
    // Scores get a key's factor, weights a value's.  A value that is no number is 0 here, so that it is nothing to rows that do not see it, and
    // its key's factor is NaN: scores of rows that do are NaN, and so is what they come to.
    auto store = [&](int buf) {
#pragma unroll
        for (int u = 0; u < LOADS; ++u)
            if (ITEMS % THREADS == 0 || tid + THREADS * u < ITEMS) {
                const int key = key_of(u), col = part_of(u);
                u32x4 x[2];
                numbers(codes[u].k, codes[u].kstep, x);
                uint8_t* k = lds + (buf * KT + key) * KPITCH + col * 32;
                *reinterpret_cast<u32x4*>(k) = x[0];
                *reinterpret_cast<u32x4*>(k + 16) = x[1];
                bool number = true;
                if constexpr (MX) {
#pragma unroll
                    for (int e = 0; e < (D / 32 + 3) / 4; ++e) number = number && !any_no_number(codes[u].vscale[e]);
                    const unsigned four = D > 128 && col >= 8 ? codes[u].vscale[(D / 32 - 1) / 4] : codes[u].vscale[0];
#pragma unroll
                    for (int e = 0; e < PIECE / 4; ++e) codes[u].v[e] = number ? codes[u].v[e] : 0u;
                    numbers(codes[u].v, number ? mx_scale_value(four >> (col / 2 % 4 * 8) & 0xFFu) : 1.0f, x);
                } else {
                    number = (__float_as_uint(codes[u].vstep) >> 23 & 0xFFu) < 0xFFu;
                    numbers(codes[u].v, 1.0f, x);
                }
                uint8_t* v = lds + 2 * KT * KPITCH + (buf * KT + key) * VPITCH + col * 32;
                *reinterpret_cast<u32x4*>(v) = x[0];
                *reinterpret_cast<u32x4*>(v + 16) = x[1];
                if (col == 0) {
                    ksteps[buf][key] = number ? (MX ? p.scale : codes[u].kstep * p.scale) : __uint_as_float(0x7FC00000u);
                    if constexpr (!MX) vsteps[buf][key] = number ? codes[u].vstep : 1.0f;
                    if ((key & 15) == 0) there_of[buf][key >> 4] = there[u];
                }
            }
    };

    f32x4 acc[DT][NT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int u = 0; u < NT; ++u) acc[t][u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float top[NT], total[NT];
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        top[u] = -__builtin_inff();
        total[u] = 0.0f;
    }
    auto use = [&](int j0, int buf) {
        unsigned groups = 0;                                // of 16 positions whose pages are there
#pragma unroll
        for (int m = 0; m < MT; ++m) groups |= (unsigned)there_of[buf][m] << m;
        groups = __builtin_amdgcn_readfirstlane(groups);
        const bool whole = j0 >= all_from && j0 + KT <= all_end && j0 + KT <= end && groups == (1u << MT) - 1;
        f32x4 s[MT][NT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
#pragma unroll
            for (int u = 0; u < NT; ++u) s[m][u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                const u32x4 k = *reinterpret_cast<const u32x4*>(lds + (buf * KT + 16 * m + fr) * KPITCH + (32 * st + 8 * fq) * 2);
#pragma unroll
                for (int u = 0; u < NT; ++u)
#pragma unroll
                    for (int e = N - 1; e >= 0; --e) s[m][u] = multiply_bf16(k, q[u][st][e], s[m][u]);
            }
            const f32x4 factor = *reinterpret_cast<const f32x4*>(&ksteps[buf][16 * m + 4 * fq]);
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[m][u][i] *= factor[i];
        }
        if (!whole) {                                       // a bit for each of four positions, without a comparison for each
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int u = 0; u < NT; ++u) {
                    const int base = j0 + 16 * m + 4 * fq, last = mine[u].from + mine[u].count < end ? mine[u].from + mine[u].count : end;
                    const int from = clamp_int(mine[u].from - base, 0, 4), to = clamp_int(last - base, 0, 4);
                    const int sees = groups >> m & 1 ? ((1 << to) - 1) & ~((1 << from) - 1) : 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const unsigned all = (unsigned)__builtin_amdgcn_sbfe(sees, i, 1);      // ones or zeros
                        s[m][u][i] = __uint_as_float((__float_as_uint(s[m][u][i]) & all) | (0xFF800000u & ~all));
                    }
                }
        }
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            float most = s[0][u][0];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) most = __builtin_fmaxf(most, s[m][u][i]);
            if (__any(most > top[u] + kSlack)) {
                const float next = __builtin_fmaxf(top[u], over_quarters_max(most));
                const float shrink = next == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(top[u] - next);
                top[u] = next;
                total[u] *= shrink;
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[t][u][i] *= shrink;
            }
        }
#pragma unroll
        for (int kk = 0; kk < MT / 2; ++kk) {
            u32x4 w[NT][NV];
#pragma unroll
            for (int u = 0; u < NT; ++u) {
                const float base = top[u] == -__builtin_inff() ? 0.0f : top[u];
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int m = 2 * kk + i / 4;
                    x[i] = __builtin_amdgcn_exp2f(s[m][u][i % 4] - base);
                    total[u] += x[i];
                }
                if constexpr (!MX) {
                    const f32x4 f[2] = {*reinterpret_cast<const f32x4*>(&vsteps[buf][32 * kk + 4 * fq]),
                                        *reinterpret_cast<const f32x4*>(&vsteps[buf][32 * kk + 16 + 4 * fq])};
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] *= f[i / 4][i % 4];
                }
                bf16_sums<NV>(x, w[u]);
            }
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                const uint8_t* v = lds + 2 * KT * KPITCH + (buf * KT + 32 * kk + 4 * fq + (fr >> 2)) * VPITCH + (16 * t + (fr & 3) * 4) * 2;
                const u32x2 lo = read_transposed(v), hi = read_transposed(v + 16 * VPITCH);
                const u32x4 vt = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
                for (int u = 0; u < NT; ++u)
#pragma unroll
                    for (int e = NV - 1; e >= 0; --e) acc[t][u] = multiply_bf16(vt, w[u][e], acc[t][u]);
            }
        }
    };

    // One barrier for KT positions: the next ones' numbers go into the other buffer while these are used.
    if (begin < end) {
        look_up(begin);
        load();
        store(0);
        look_up(begin + KT);
        __syncthreads();
        int buf = 0;
        for (int j = begin; j < end; j += KT, buf ^= 1) {
            const bool more = j + KT < end;
            if (more) {
                load();
                look_up(j + 2 * KT);                        // (a table's entry has as long as the codes to come)
            }
            if (j < wave_end && j + KT > wave_from) use(j, buf);
            if (more) store(buf ^ 1);
            __syncthreads();
        }
    }
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        const float sum = over_quarters_sum(total[u]);
        if (wave_row + 16 * u + fr >= rows) continue;
        const int64_t out_row = (int64_t)(t0 + token[u]) * p.Hq + head[u];
        if (p.parts > 1) {
            const int64_t to = part * ((int64_t)p.s.T * p.Hq) + out_row;
            if (fq == 0) {
                p.stats[2 * to] = top[u];
                p.stats[2 * to + 1] = sum;
            }
#pragma unroll
            for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4*>(p.sums + to * D + 16 * t + 4 * fq) = acc[t][u];
            continue;
        }
        if (p.lse && fq == 0)
            p.lse[out_row] = sum > 0.0f ? (top[u] + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f : (sum == 0.0f ? -__builtin_inff() : sum);
        elem_t<T>* y = static_cast<elem_t<T>*>(p.Y) + (int64_t)(t0 + token[u]) * p.ldy + head[u] * p.hdy + 4 * fq;
        const float share = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v = sum == 0.0f ? 0.0f : acc[t][u][i] * share;
                if (p.c.vdepth) v *= cache_doublings(p.c.vdepth[h * D + 16 * t + 4 * fq + i]);
                y[16 * t + i] = float_to_elem<T>(v);
            }
    }
}

// Most parts: what a weight each fits in LDS for.
constexpr int kMostParts = 2048;

// The parts of a row put together, one workgroup per row: every wave finds the parts' common maximum, 64 parts to a look, and their weights
// meet in LDS; then their columns, four to a lane, as many parts at once as there are lanes for, the first of them asked for ahead.
template <Elem T, int D>
__global__ __launch_bounds__(256) void attend_join_kernel(Attention p) {
    __shared__ float weight[kMostParts];
    __shared__ f32x4 partial[256];
    constexpr int AHEAD = 4;
    constexpr int lanes = D / 4, groups = 256 / lanes;
    const int64_t rows = (int64_t)p.s.T * p.Hq, row = blockIdx.x;
    const int t = (int)(blockIdx.x / (unsigned)p.Hq), head = (int)(blockIdx.x % (unsigned)p.Hq), tid = (int)threadIdx.x, lane = tid & 63;
    const int group = tid / lanes, d = tid % lanes * 4;
    auto columns = [&](int k) { return *reinterpret_cast<const f32x4*>(p.sums + (k * rows + row) * D + d); };
    const int past = p.s.cu[p.s.B];
    f32x4 first[AHEAD];                                     // (of parts without a position: not written, and not used)
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (group < groups && group + i * groups < p.parts) first[i] = columns(group + i * groups);
    float all = -__builtin_inff();
    for (int i = lane; i < p.parts; i += 64) all = __builtin_fmaxf(all, p.stats[2 * (i * rows + row)]);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) all = __builtin_fmaxf(all, __shfl_xor(all, m));
    const float base = all == -__builtin_inff() ? 0.0f : all;
    float sum = 0.0f;
    for (int i = lane; i < p.parts; i += 64) {
        const float total = p.stats[2 * (i * rows + row) + 1];
        // below 0: a part without positions, which is left out; any other counts, if only by 0, so that a NaN among its values stays one
        const float f = total == 0.0f ? -1.0f : __builtin_amdgcn_exp2f(p.stats[2 * (i * rows + row)] - base);
        if (total != 0.0f) sum += total * f;
        weight[i] = f;                                      // (by every wave, the same)
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) sum += __shfl_xor(sum, m);
    __syncthreads();
    if (t >= past) return;                                  // behind the last sequence
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    auto add = [&](const f32x4& x, float w) {
        if (!(w < 0.0f))                                    // (NaN is not below 0)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += x[e] * w;
    };
    if (group < groups) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (group + i * groups < p.parts) add(first[i], weight[group + i * groups]);
#pragma unroll 4
        for (int k = group + AHEAD * groups; k < p.parts; k += groups) {
            const float w = weight[k];
            if (!(w < 0.0f)) add(columns(k), w);
        }
    }
    partial[tid] = v;
    __syncthreads();
    if (tid >= lanes) return;
    for (int g = 1; g < groups; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += partial[g * lanes + tid][e];
    elem_t<T>* y = static_cast<elem_t<T>*>(p.Y) + t * p.ldy + head * p.hdy + d;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float o = sum == 0.0f ? 0.0f : v[e] / sum;
        if (p.c.vdepth) o *= cache_doublings(p.c.vdepth[head / p.G * D + d + e]);
        y[e] = float_to_elem<T>(o);
    }
    if (p.lse && tid == 0) p.lse[row] = sum > 0.0f ? (all + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f : (sum == 0.0f ? -__builtin_inff() : sum);
}

struct AttentionPlan {
    bool many;                              // rows: the kernel with tiles of them
    int64_t tiles;
    int parts;
    int64_t chunk;
};

// Which kernel, and parts of the positions where the tiles alone leave compute units idle.
//
// Tiles of many rows from five eighths of one to a sequence on, by the call's mean (us, 16 rows a workgroup / tiles; 8 bits, bf16, sequences of an
// eighth of the longest on).  A call that mixes prompts with single tokens goes one way altogether.
//   rows:                            48             64             80             96            128
//   64 to 8192, 4 heads of 128   195 / 186      196 / 196      254 / 216      265 / 202      324 / 258
//   64, in 4 bits                143 / 179      151 / 189      198 / 214      205 / 196      239 / 248
//   64 to 1024                  52.7 / 61.2    57.6 / 66.7    74.3 / 73.6    79.5 / 79.2    60.9 / 81.2
//   16 to 2048, heads of 256    55.5 / 37.5    54.0 / 43.2    67.0 / 63.2    62.8 / 57.9    76.1 / 57.7
// Workgroups a compute unit: 2 of up to three sequences, whose parts the join has to read, 8 of more, whose lengths differ (us, 2 / 4 / 8; 8 bits, 8
// heads of 128, 4 queries each): one of 100003 41.7 / 47.8 / 51.8, two of 100000 82.7 / 91.1 / 90.8, three to 60000 51.0 / 50.3 / 53.6, 8 to 30000
// 77.1 / 63.1 / 64.1, 64 to 8192 149 / 142 / 136.
static AttentionPlan plan_attention(int64_t T, int64_t B, int64_t H, int64_t Hq, int64_t D, int64_t most, int64_t window) {
    const int64_t G = Hq / H, cus = compute_units(), range = window > 0 && window + T < most ? window + T : most;
    const int64_t tile_rows = D <= 128 ? 128 : 64;
    const bool many = 8 * T * G >= 5 * tile_rows * B;
    const int64_t rows = many ? tile_rows : 16, tiles = T * G / rows + B, per_cu = B < 4 ? 2 : 8;
    AttentionPlan a{many, tiles, 1, 0};
    const int64_t want = ceil_div(per_cu * cus, tiles * H), can = ceil_div(range, 32 * kAttendWaves * 2), fit = ((int64_t)48 << 20) / (T * Hq * (D + 2) * 4);
    int64_t parts = want < can ? want : can;
    parts = parts < fit ? parts : fit;
    parts = parts < kMostParts ? parts : kMostParts;
    if (parts > 1) {
        a.chunk = round_up(ceil_div(range + 31, parts), 32 * kAttendWaves);
        parts = ceil_div(range + 31, a.chunk);
    }
    a.parts = parts > 1 ? (int)parts : 1;
    return a;
}

size_t cache_attention_workspace_bytes(int64_t T, int64_t B, int64_t H, int64_t Hq, int64_t D, int64_t most, int64_t window) {
    const AttentionPlan a = plan_attention(T, B, H, Hq, D, most, window);
    return a.parts > 1 ? (size_t)a.parts * (size_t)(T * Hq) * (size_t)(D + 2) * 4 : 0;
}

template <Elem T, CacheFormat F, int D>
static hipError_t run_attention(const Attention& p, const AttentionPlan& a, hipStream_t stream) {
    const dim3 grid((unsigned)(a.tiles * p.c.H * p.parts));
    hipError_t e;
    if (a.many) {
        constexpr int LDS = AttendTile<T, D>::LDS;
        if constexpr (LDS > 65536) {
            static std::atomic<bool> allowed[kMaxDevices];
            e = allow_lds(reinterpret_cast<const void*>(&attend_tile_kernel<T, F, D>), LDS, allowed);
            if (e != hipSuccess) return e;
        }
        e = launch_kernel(kTimeGemm, attend_tile_kernel<T, F, D>, grid, dim3(AttendTile<T, D>::THREADS), (unsigned)LDS, stream, p);
    } else {
        e = launch_kernel(kTimeGemm, attend_rows_kernel<T, F, D>, grid, dim3(kAttendWaves * 64), 0, stream, p);
    }
    if (e != hipSuccess || p.parts == 1) return e;
    return launch_kernel(0, attend_join_kernel<T, D>, dim3((unsigned)((int64_t)p.s.T * p.Hq)), dim3(256), 0, stream, p);
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
    const AttentionPlan a = plan_attention(s.T, s.B, c.H, Hq, c.D, most, window);
    float* sums = static_cast<float*>(workspace);
    const int64_t held = most < c.cols * c.P ? most : c.cols * c.P;
    Attention p{c, s, Q, ldq, hdq, Hq, Hq / c.H, scale * 1.44269504088896341f, (int)(window < 0x7FFFFFFF ? window : 0), (int)held,
                (unsigned)(((uint64_t)1 << 32) / c.P) + 1, Y, ldy, hdy, lse, (int)a.tiles, a.parts, (int)a.chunk, sums, nullptr};
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
