// Scoring of tokens: log probabilities of given tokens, entropy and the most likely alternatives of rows of logits.
//
// One pass over a row: every lane keeps the running maximum m of what it has seen, s = sum exp(x - m) and
// w = sum (x - m) exp(x - m); where the maximum grows by d, s -> s e^-d and w -> e^-d (w - d s).  Joined over the row,
// log p(t) = (x_t - m) - log s and the entropy is log s - w / s (both free of the cancellation of sum p log p).
// The alternatives come out of the same pass: the k-th largest of 64 groups' maxima is a bound that at least k logits
// reach, only the lanes that reach it hold any of them, and only those lanes' pieces of the row are looked through again.
// Bound by HBM for many rows (4096 x 100003 bf16 144 us, 5.7 TB/s; 700 x 33001 fp32 18, 5.1), by latency for few: of 1 x 33001's 6.8 us
// the exponentials of 33 logits a lane on one compute unit take 3, the loads 1, bound and list 1, the ranking 1.  All sums are in fp32.
#include "row_types.h"

namespace ocs {

constexpr int kTopGroups = 256;       // maxima of lanes, or of quads of them, that are held against the bound
constexpr int kTopList = 1024;        // logits that may reach it; more are selected one by one, each a pass over the row:
                                      // rows of equal values, and few rows of logits that fall from token to token (see bound_of)
constexpr float kLowest = -3.402823466e+38f;
constexpr float kLog2e = 1.44269504f;

struct TokenRows {
    const void* logits;
    int64_t ld;
    int V, k;
    const int32_t* tokens;
    float* logprob;
    float* entropy;
    int32_t* top_ids;
    float* top_logprobs;
    // rows shared by several workgroups: part_len logits each, sums [rows][parts][4], keys [rows][parts][k]
    int parts, part_len;
    float* sums;
    unsigned long long* keys;
};

// Logits as whole numbers that order like them: -0 with +0, NaN above everything, 0 below everything.  Nothing is 0xFFFFFFFF: every key
// is below ~0, which is what a selection begins below.
__device__ __forceinline__ unsigned order_of(float v) {
    if (v != v) return 0xFFFFFFFEu;
    const unsigned b = __float_as_uint(v + 0.0f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned o) {
    return __uint_as_float((o & 0x80000000u) ? o & 0x7FFFFFFFu : ~o);
}
// value, then lowest index
__device__ __forceinline__ unsigned long long key_of(float v, int index) {
    return ((unsigned long long)order_of(v) << 32) | (0xFFFFFFFFu - (unsigned)index);
}
__device__ __forceinline__ int index_of(unsigned long long key) { return (int)(0xFFFFFFFFu - (unsigned)key); }

__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// The sum over the 64 lanes of a wave, the same in all of them (rows of 16 lanes by DPP, then the four rows).
__device__ __forceinline__ float wave_sum(float v) {
    v += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0xB1, 0xF, 0xF, false));    // quad_perm [1,0,3,2]
    v += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x4E, 0xF, 0xF, false));    // quad_perm [2,3,0,1]
    v += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x141, 0xF, 0xF, false));   // row_half_mirror
    v += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x140, 0xF, 0xF, false));   // row_mirror
    const float a = __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(v), 0));
    const float b = __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(v), 16));
    const float c = __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(v), 32));
    const float d = __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(v), 48));
    return (a + b) + (c + d);
}

struct Running {
    float m = kLowest, s = 0.0f, w = 0.0f;
};

// What s and w become when the maximum goes from m to top.
__device__ __forceinline__ void raise(Running& r, float top) {
    const float d = fmaxf(r.m - top, -150.0f);      // e^-150 is zero in fp32, and 0 * -150 is
    const float f = exp_of(d);
    r.w = f * __builtin_fmaf(r.s, d, r.w);
    r.s *= f;
    r.m = top;
}

__device__ __forceinline__ void join_wave(Running& r) {
    raise(r, value_of(wave_umax32(order_of(r.m))));
    r.s = wave_sum(r.s);
    r.w = wave_sum(r.w);
}

// KNOWN: r.m is at least every one of the logits already.
template <bool KNOWN = false, int N>
__device__ __forceinline__ void add_logits(Running& r, const float (&v)[N]) {
    if constexpr (!KNOWN) {
        float top = r.m;
#pragma unroll
        for (int e = 0; e < N; ++e) top = fmaxf(top, v[e]);
        if (top > r.m) raise(r, top);
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float d = v[e] - r.m;                 // -inf for a token ruled out, NaN stays NaN
        const float x = exp_of(d);
        r.s += x;
        r.w = __builtin_fmaf(fmaxf(d, -150.0f), x, r.w);
    }
}

template <Elem T, bool KNOWN = false>
__device__ __forceinline__ void add_piece(Running& r, u32x4 raw) {
    float v[kVec<T>];
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) v[e] = piece_elem<T>(raw, e);
    add_logits<KNOWN>(r, v);
}

// What a row comes to.
struct RowResult {
    float m, log_s;
    bool bad;                                       // NaN or +inf in the row
};
__device__ __forceinline__ RowResult result_of(const Running& r) {
    const bool none = r.m == kLowest && r.s == 0.0f;               // every token ruled out
    return {r.m, none ? 0.0f : logf(r.s), !(r.s < 3.402823466e+38f)};
}
__device__ __forceinline__ void write_row(const TokenRows& p, int64_t row, const Running& r, const RowResult& q, float given,
                                          bool has_token) {
    const float nan = __uint_as_float(0x7FC00000u);
    if (p.logprob) p.logprob[row] = !has_token ? 0.0f : q.bad ? nan : (given - q.m) - q.log_s;
    if (p.entropy) p.entropy[row] = q.bad ? nan : r.s == 0.0f ? 0.0f : q.log_s - r.w / r.s;
}
__device__ __forceinline__ void write_top(const TokenRows& p, int64_t row, const RowResult& q, int i, unsigned long long key) {
    p.top_ids[row * p.k + i] = index_of(key);
    p.top_logprobs[row * p.k + i] = q.bad ? __uint_as_float(0x7FC00000u) : (value_of((unsigned)(key >> 32)) - q.m) - q.log_s;
}

constexpr unsigned kFirstFinite = 0x00800000u;      // order_of(kLowest): what is below is -inf or nothing

// A number that at least k of the wave's keys (4 a lane) reach: the k-th largest of the lanes' maxima, to its upper 16 bits.  A lane's four
// groups are neighbours in the row, so it is a weak bound where large logits are (us, k = 5 / 20 / 32, of shuffled logits, of -log rank + N(0, 1)
// in order of rank, of -log rank alone, of equal ones: 1 x 33001 fp32 6.4 / 6.9 / 7.2, 6.6 / 8.2 / 11.0, 9.7 / 114 / 178, 40 / 121 / 186;
// 700 x 33001 bf16 12.9 / 14.2 / 15.7, 14.2 / 20.4 / 25.2, 17.8 / 53 / 100, 290 / 933 / 1441).
__device__ __forceinline__ unsigned bound_of(u32x4 keys, int k) {
    unsigned most = keys[0];
#pragma unroll
    for (int e = 1; e < 4; ++e) most = keys[e] > most ? keys[e] : most;
    unsigned bound = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const unsigned next = bound | (1u << bit);
        bound = (int)__popcll(__ballot(most >= next)) >= k ? next : bound;
    }
    return bound;
}

typedef unsigned long long u64x2 __attribute__((ext_vector_type(2)));

template <int NT, bool HELD>
struct TopShared {
    alignas(16) unsigned group[kTopGroups];
    float wave_m[NT / 64], wave_s[NT / 64], wave_w[NT / 64];
    alignas(16) unsigned long long list[kTopList];
    unsigned long long top[32];
    unsigned long long wave_key[NT / 64];
    int reach[HELD ? 1 : NT / 64][kTopGroups];                     // (a list per wave)
    int list_n;
};

template <Elem T>
constexpr unsigned kNoLogits = T == Elem::f32 ? 0xFF800000u : T == Elem::bf16 ? 0xFF80FF80u : 0xFC00FC00u;   // -inf

// NT lanes per row (or part of a row).  HELD: the row's pieces stay in registers, U a lane; otherwise they pass through, U requested
// ahead of the U that are added up.
template <Elem T, int NT, int U, bool HELD>
__global__ __launch_bounds__(NT) void token_rows_kernel(TokenRows p) {
    constexpr int VEC = kVec<T>;
    constexpr int GW = NT / kTopGroups;                            // lanes of a group
    static_assert(GW == 1 || GW == 2 || GW == 4, "a lane, a pair or a quad");
    __shared__ TopShared<NT, HELD> sh;
    const int tid = (int)threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row = p.parts == 1 ? (int64_t)blockIdx.x : (int64_t)(blockIdx.x / (unsigned)p.parts);
    const int part = p.parts == 1 ? 0 : (int)(blockIdx.x - (unsigned)row * (unsigned)p.parts);
    const elem_t<T>* whole = static_cast<const elem_t<T>*>(p.logits) + row * p.ld;
    const int first = part * p.part_len;
    const int n = p.V - first < p.part_len ? p.V - first : p.part_len;
    const elem_t<T>* x = whole + first;

    // pieces at 16-byte addresses; what lies before and behind them, at most VEC - 1 logits each, one lane each
    int head = (int)((16u - ((unsigned)(uintptr_t)x & 15u)) & 15u) / (int)sizeof(elem_t<T>);
    head = head < n ? head : n;
    const int body = (n - head) / VEC, rest = n - head - body * VEC;
    const elem_t<T>* xb = x + head;
    int edge = -1;                                                 // this lane's single logit
    if (tid < head) edge = tid;
    else if (tid >= VEC && tid - VEC < rest) edge = head + body * VEC + tid - VEC;

    int token = -1;                                                // asked for first: a wait for it is no wait for the row
    if (p.parts == 1 && p.tokens != nullptr) token = p.tokens[row];
    u32x4 raw[U];
    if constexpr (HELD) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw[u] = u32x4{kNoLogits<T>, kNoLogits<T>, kNoLogits<T>, kNoLogits<T>};
            if (u * NT + tid < body) raw[u] = load_piece<T>(xb + (u * NT + tid) * VEC);
        }
    }
    float edge_v = -__builtin_inff();
    if (edge >= 0) edge_v = elem_to_float<T>(x[edge]);
    if (tid == 0) sh.list_n = 0;

    Running r;
    if constexpr (HELD) {
        float top = fmaxf(kLowest, edge_v);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < VEC; ++e) top = fmaxf(top, piece_elem<T>(raw[u], e));
        r.m = top;
#pragma unroll
        for (int u = 0; u < U; ++u) add_piece<T, true>(r, raw[u]);
    } else {
        int i0 = 0;
        if (NT * U <= body) {
            u32x4 next[U];
#pragma unroll
            for (int u = 0; u < U; ++u) next[u] = load_piece<T>(xb + (int64_t)(u * NT + tid) * VEC);
            for (; i0 + NT * U <= body; i0 += NT * U) {
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u] = next[u];
                if (i0 + 2 * NT * U <= body) {
#pragma unroll
                    for (int u = 0; u < U; ++u) next[u] = load_piece<T>(xb + (int64_t)(i0 + (U + u) * NT + tid) * VEC);
                }
                float v[U * VEC];
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) v[u * VEC + e] = piece_elem<T>(raw[u], e);
                add_logits(r, v);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + u * NT + tid < body) raw[u] = load_piece<T>(xb + (int64_t)(i0 + u * NT + tid) * VEC);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + u * NT + tid < body) add_piece<T>(r, raw[u]);
    }
    if (edge >= 0) {
        const float v[1] = {edge_v};
        add_logits(r, v);
    }

    if (token < 0 || token >= p.V) token = -1;
    float given = 0.0f;
    if (token >= 0) given = elem_to_float<T>(whole[token]);

    // each wave's maximum and sums, and the lanes' maxima (0: nothing but -inf)
    const unsigned mine = r.s == 0.0f ? 0u : order_of(r.m);
    {
        unsigned g = mine;
        if constexpr (GW >= 2) {
            const unsigned other = (unsigned)__builtin_amdgcn_update_dpp(0, (int)g, 0xB1, 0xF, 0xF, false);   // quad_perm [1,0,3,2]
            g = other > g ? other : g;
        }
        if constexpr (GW == 4) {
            const unsigned other = (unsigned)__builtin_amdgcn_update_dpp(0, (int)g, 0x4E, 0xF, 0xF, false);            // quad_perm [2,3,0,1]
            g = other > g ? other : g;
        }
        if (tid % GW == 0) sh.group[tid / GW] = g;
        join_wave(r);
        if (lane == 0) {
            sh.wave_m[wave] = r.m;
            sh.wave_s[wave] = r.s;
            sh.wave_w[wave] = r.w;
        }
    }
    __syncthreads();
    r = Running{};
    if (lane < NT / 64) {
        r.m = sh.wave_m[lane];
        r.s = sh.wave_s[lane];
        r.w = sh.wave_w[lane];
    }
    join_wave(r);                                                  // the row's, in every wave
    if (tid == 0 && p.parts > 1) {
        float* to = p.sums + ((int64_t)row * p.parts + part) * 4;
        to[0] = r.m;
        to[1] = r.s;
        to[2] = r.w;
    }
    if (p.k == 0) {
        if (tid == 0 && p.parts == 1) write_row(p, row, r, result_of(r), given, token >= 0);
        return;
    }

    const bool odd = !(r.s < 3.402823466e+38f);                    // NaN or +inf: the maxima do not show them all
    const int want = p.k < n ? p.k : n;
    if (!odd) {
        const u32x4 groups = *reinterpret_cast<const u32x4*>(&sh.group[4 * lane]);
        const unsigned reached = bound_of(groups, p.k), bound = reached > kFirstFinite ? reached : kFirstFinite;
        const float least = value_of(bound);
        auto offer = [&](float v, int index) {
            const int at = atomicAdd(&sh.list_n, 1);
            if (at < kTopList) sh.list[at] = key_of(v, first + index);
        };
        if (edge >= 0 && edge_v >= least) offer(edge_v, edge);
        if constexpr (HELD) {
            // which of the lane's logits reach it, then those few once more (short code: a row's is fetched for that row alone)
            static_assert(U * VEC <= 64, "a bit per logit");
            if (mine >= bound) {
                unsigned hits[2] = {0u, 0u};
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        hits[(u * VEC + e) / 32] |= piece_elem<T>(raw[u], e) >= least ? 1u << ((u * VEC + e) % 32) : 0u;
                unsigned long long in = ((unsigned long long)hits[1] << 32) | hits[0];
                for (; in != 0; in &= in - 1) {
                    const int b = (int)__ffsll(in) - 1, index = head + (b / VEC * NT + tid) * VEC + b % VEC;
                    offer(elem_to_float<T>(x[index]), index);
                }
            }
        } else {
            // the groups that reach the bound (group 4 l + e is lane l's key e), listed by every wave alike, then the pieces of them all
            int reach_n = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned long long in = __ballot(groups[e] >= bound);
                if (groups[e] >= bound) sh.reach[wave][reach_n + (int)__popcll(in & ((1ull << lane) - 1ull))] = 4 * lane + e;
                reach_n += (int)__popcll(in);
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            const unsigned each = (unsigned)(body + NT - 1) / NT * GW, all = (unsigned)reach_n * each;
            for (unsigned j = (unsigned)tid; j < all; j += NT) {
                const unsigned a = j / each, in = j - a * each, i = in / GW * NT + (unsigned)sh.reach[wave][a] * GW + in % GW;
                if ((int)i >= body) continue;
                const u32x4 again = load_piece<T>(xb + (int64_t)i * VEC);
                unsigned hits = 0;
#pragma unroll
                for (int e = 0; e < VEC; ++e) hits |= piece_elem<T>(again, e) >= least ? 1u << e : 0u;
                for (; hits != 0; hits &= hits - 1) {
                    const int index = head + (int)i * VEC + __ffs((int)hits) - 1;
                    offer(elem_to_float<T>(x[index]), index);
                }
            }
        }
    }
    __syncthreads();
    int got = sh.list_n;
    if (odd || got > kTopList) {
        // one by one, from the largest down, each the largest key below the last
        unsigned long long last = ~0ull;
        for (int i = 0; i < want; ++i) {
            unsigned long long best = 0;
            for (int j = tid; j < n; j += NT) {
                const unsigned long long key = key_of(elem_to_float<T>(x[j]), first + j);
                best = key < last && key > best ? key : best;
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) {
                const unsigned long long other = __shfl_xor(best, o);
                best = other > best ? other : best;
            }
            if (lane == 0) sh.wave_key[wave] = best;
            __syncthreads();
            best = sh.wave_key[0];
#pragma unroll
            for (int w = 1; w < NT / 64; ++w) best = sh.wave_key[w] > best ? sh.wave_key[w] : best;
            if (tid == 0) sh.top[i] = best;
            last = best;
            __syncthreads();
        }
        if (wave != 0) return;
    } else {
        // a list of a wave's size or less, most of the time: the first wave has the rest
        if (got > 64) {
            for (int i = tid; i < got; i += NT) {
                const unsigned long long key = sh.list[i];
                int ahead = 0;
                for (int j = 0; j < got; ++j) ahead += sh.list[j] > key ? 1 : 0;
                if (ahead < want) sh.top[ahead] = key;
            }
            __syncthreads();
            if (wave != 0) return;
        } else {
            if (wave != 0) return;
            // every lane counts the keys above its own, eight at a time from LDS (k = 20, some 50 keys: 1.5 us less than one by one out of
            // the lanes); what follows the list reads as zero
            if (lane >= got) sh.list[lane] = 0ull;
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            const unsigned long long key = sh.list[lane];
            int ahead = 0;
            for (int j = 0; j < got; j += 8) {
                u64x2 other[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) other[q] = *reinterpret_cast<const u64x2*>(&sh.list[j + 2 * q]);
#pragma unroll
                for (int q = 0; q < 4; ++q) ahead += (other[q][0] > key ? 1 : 0) + (other[q][1] > key ? 1 : 0);
            }
            if (lane < got && ahead < want) sh.top[ahead] = key;
        }
        // fewer finite logits than alternatives: then all others are -inf, and the first of them follow
        for (int j0 = 0; got < want && j0 < n; j0 += 64) {
            const float v = j0 + lane < n ? elem_to_float<T>(x[j0 + lane]) : 0.0f;
            const bool out = j0 + lane < n && v == -__builtin_inff();
            const unsigned long long mask = __ballot(out);
            const int at = got + (int)__popcll(mask & ((1ull << lane) - 1ull));
            if (out && at < want) sh.top[at] = key_of(v, first + j0 + lane);
            got += (int)__popcll(mask);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    if (p.parts == 1) {
        const RowResult q = result_of(r);
        if (tid == 0) write_row(p, row, r, q, given, token >= 0);
        if (tid < p.k) write_top(p, row, q, tid, sh.top[tid]);
    } else if (tid < p.k) {
        p.keys[((int64_t)row * p.parts + part) * p.k + tid] = tid < want ? sh.top[tid] : 0ull;   // (a part shorter than k)
    }
}

// The parts of a row joined by one wave, a lane per part: sums at the row's maximum, and the lists, each in order, merged.
constexpr int kMostParts = 64;
template <Elem T>
__global__ __launch_bounds__(64) void token_join_kernel(TokenRows p) {
    __shared__ unsigned long long keys[kMostParts * 33];           // a list's end: 0
    const int lane = (int)threadIdx.x;
    const int64_t row = blockIdx.x;
    const unsigned long long* from = p.keys + (int64_t)row * p.parts * p.k;
    for (int i = lane; i < p.parts * p.k; i += 64) keys[(i / p.k) * 33 + i % p.k] = from[i];
    for (int i = lane; i < p.parts; i += 64) keys[i * 33 + p.k] = 0ull;
    int token = -1;
    float given = 0.0f;
    if (p.tokens != nullptr) {
        token = p.tokens[row];
        if (token < 0 || token >= p.V) token = -1;
        if (token >= 0) given = elem_to_float<T>((static_cast<const elem_t<T>*>(p.logits) + row * p.ld)[token]);
    }
    Running r;
    if (lane < p.parts) {
        const float* sums = p.sums + ((int64_t)row * p.parts + lane) * 4;
        r.m = sums[0];
        r.s = sums[1];
        r.w = sums[2];
    }
    join_wave(r);
    const RowResult q = result_of(r);
    if (lane == 0) write_row(p, row, r, q, given, token >= 0);
    __syncthreads();
    const unsigned long long* mine = keys + lane * 33;
    unsigned long long next = lane < p.parts ? mine[0] : 0ull;
    unsigned long long best_of_i = 0ull;                           // lane i keeps the i-th
    for (int i = 0; i < p.k; ++i) {
        const unsigned hi = wave_umax32((unsigned)(next >> 32));
        const unsigned lo = wave_umax32((unsigned)(next >> 32) == hi ? (unsigned)next : 0u);
        const unsigned long long best = ((unsigned long long)hi << 32) | lo;
        if (lane == i) best_of_i = best;
        if (next == best && best != 0ull) next = *++mine;          // (keys differ: one lane)
    }
    if (lane < p.k) write_top(p, row, q, lane, best_of_i);
}

// Logits that 1024 lanes hold, whatever their type: 16 pieces a lane of fp32, 8 of the others.
constexpr int kHeldLogits = 65536;
constexpr int64_t kMostPartRows = 2048;   // parts of all rows together: the workspace stays below a megabyte

struct TokenPlan {
    int parts, part_len;
    size_t keys_off, total;
};
// Rows that fill the chip have a workgroup each.  Fewer ones, longer than a workgroup holds, are cut into parts of half of what it does: the
// exponentials of a lane's logits are what a part takes longest over (bf16, us from a graph, parts of 65536 / 32768 / 16384 / 8192: 1 x 100003
// 11.7 / 9.8 / 9.6 / 9.7, 64 x 100003 13.8 / 11.4 / 11.9 / 14.6, 250 x 70001 22.6 / 18.0 / 16.7 / 20.4, 64 x 250001 15.4 / 15.2 / 15.7 / 20.9).
constexpr int kPartLogits = 32768;
static TokenPlan plan_token_rows(int64_t M, int64_t V, int k) {
    TokenPlan t{1, (int)V, 0, 0};
    if (M <= compute_units() && M <= kMostPartRows / 2 && V > kHeldLogits) {
        int64_t parts = ceil_div(V, kPartLogits);
        const int64_t most = kMostPartRows / M < kMostParts ? kMostPartRows / M : kMostParts;
        parts = parts < most ? parts : most;
        t.part_len = (int)round_up(ceil_div(V, parts), 64);
        t.parts = (int)ceil_div(V, t.part_len);
        t.keys_off = (size_t)round_up(M * t.parts * 16, 256);
        t.total = t.keys_off + (size_t)M * t.parts * k * 8;
    }
    return t;
}
size_t token_logprobs_workspace_bytes(int64_t M, int64_t V, int k) { return plan_token_rows(M, V, k).total; }

// One launch for every kMostLanes lanes' worth of rows: as a rule all of them, rows in parts always (there are few).
template <Elem T, int NT, int U, bool HELD>
static hipError_t run_token_kernel(TokenRows p, int64_t M, hipStream_t stream) {
    const int64_t most = kMostLanes / NT / p.parts;
    for (int64_t left = M; left > 0;) {
        const int64_t rows = left < most ? left : most;
        const hipError_t e = launch_kernel(0, token_rows_kernel<T, NT, U, HELD>, dim3((unsigned)(rows * p.parts)), dim3(NT), 0, stream, p);
        if (e != hipSuccess) return e;
        left -= rows;
        p.logits = static_cast<const elem_t<T>*>(p.logits) + rows * p.ld;
        if (p.tokens) p.tokens += rows;
        if (p.logprob) p.logprob += rows;
        if (p.entropy) p.entropy += rows;
        if (p.k) {
            p.top_ids += rows * p.k;
            p.top_logprobs += rows * p.k;
        }
    }
    return hipSuccess;
}

// fp32 rows that 1024 lanes hold: 4, 9 or 16 pieces a lane.  A piece costs its exponentials whether the row fills it or not, 0.2-0.3 us.  9
// serves rows of 16385 to 36864 logits; 8 would save 0.3-0.4 us up to 32768 and send those above to 16 pieces, 2 us more; 12 would cost
// 0.6-0.8 us up to 36864 and save 1 us from there to 49152 (us, 20 alternatives, 1 row / 250 rows, by pieces a lane):
//   32000 logits   8: 6.5 / 8.1    9: 6.8 / 8.5   10: 7.1 / 8.7    12: 7.6 / 9.2
//   33001                          9: 6.8 / 8.9   10: 7.3 / 9.1    12: 7.4 / 9.6    16: 9.2 / 11.0
//   40000                                         10: 7.2 / 10.5   12: 7.7 / 10.8   16: 8.9 / 11.7
//
// Rows of up to 2048 pieces are held by 256 lanes.  Longer ones: while every row can have a compute unit to itself, by 1024 (1 x 33001
// fp32 7.0 us with 20 alternatives, 6.2 with 5; passing through 256 lanes, with the row's second look from memory, 19 where this took 8.1), otherwise they pass through 256 lanes, or 512 where
// rows come in several rounds and the last one's length counts (us, 256 / 512 lanes: 700 x 33001 fp32 18.7 / 19.2, bf16 14.2 / 14.9; 3000
// x 33001 fp32 73 / 70; 4096 x 100003 bf16 160 / 155).
template <Elem T>
static hipError_t run_token_rows(const TokenRows& p, int64_t M, hipStream_t stream) {
    const int64_t pieces = p.part_len / kVec<T>;
    hipError_t e;
    if (pieces <= 256 * 2) e = run_token_kernel<T, 256, 2, true>(p, M, stream);
    else if (pieces <= 256 * 8) e = run_token_kernel<T, 256, 8, true>(p, M, stream);
    else if (M > 4 * compute_units()) e = run_token_kernel<T, 512, 4, false>(p, M, stream);
    else if (M > compute_units() || p.part_len > kHeldLogits) e = run_token_kernel<T, 256, 4, false>(p, M, stream);
    else if (pieces <= 1024 * 4) e = run_token_kernel<T, 1024, 4, true>(p, M, stream);
    else if (T == Elem::f32 && pieces > 1024 * 9) e = run_token_kernel<T, 1024, T == Elem::f32 ? 16 : 8, true>(p, M, stream);
    else e = run_token_kernel<T, 1024, T == Elem::f32 ? 9 : 8, true>(p, M, stream);
    if (e != hipSuccess || p.parts == 1) return e;
    return launch_kernel(0, token_join_kernel<T>, dim3((unsigned)M), dim3(64), 0, stream, p);
}

hipError_t launch_token_logprobs(const void* logits, int type, int64_t M, int64_t V, int64_t ld, const int32_t* tokens, int k,
                                 float* logprob, float* entropy, int32_t* top_ids, float* top_logprobs, void* workspace,
                                 hipStream_t stream) {
    const TokenPlan t = plan_token_rows(M, V, k);
    char* base = static_cast<char*>(workspace);
    const TokenRows p{logits, ld, (int)V, k, tokens, logprob, entropy, top_ids, top_logprobs, t.parts, t.part_len,
                      t.parts > 1 ? reinterpret_cast<float*>(base) : nullptr,
                      t.parts > 1 ? reinterpret_cast<unsigned long long*>(base + t.keys_off) : nullptr};
    switch (static_cast<Elem>(type)) {
        case Elem::f32: return run_token_rows<Elem::f32>(p, M, stream);
        case Elem::bf16: return run_token_rows<Elem::bf16>(p, M, stream);
        case Elem::f16: return run_token_rows<Elem::f16>(p, M, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace ocs
