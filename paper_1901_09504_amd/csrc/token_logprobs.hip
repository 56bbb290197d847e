// Scoring of tokens: log probabilities of given tokens, entropy and the most likely alternatives of rows of logits.
//
// One pass over a row: every lane keeps the running maximum m of what it has seen, s = sum exp(x - m) and
// w = sum (x - m) exp(x - m); where the maximum grows by d, s -> s e^-d and w -> e^-d (w - d s).  Joined over the row,
// log p(t) = (x_t - m) - log s and the entropy is log s - w / s (both free of the cancellation of sum p log p).
// The alternatives come out of the same pass: the k-th largest of 256 lane maxima is a bound that at least k logits
// reach, only the lanes that reach it hold any of them, and only those lanes' pieces of the row are looked through again.
// Bound by HBM for many rows, by latency for few.  All sums are in fp32.
#include "row_types.h"

namespace ocs {

constexpr int kTopGroups = 256;       // lane maxima that the bound is taken from
constexpr int kTopList = 1024;        // logits that may reach it; more (rows of equal values) are selected one by one
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

// Logits as whole numbers that order like them: -0 with +0, NaN above everything, 0 below everything.
__device__ __forceinline__ unsigned order_of(float v) {
    if (v != v) return 0xFFFFFFFFu;
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

template <int N>
__device__ __forceinline__ void add_logits(Running& r, const float (&v)[N]) {
    float top = r.m;
#pragma unroll
    for (int e = 0; e < N; ++e) top = fmaxf(top, v[e]);
    if (top > r.m) raise(r, top);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float d = v[e] - top;                 // -inf for a token ruled out, NaN stays NaN
        const float x = exp_of(d);
        r.s += x;
        r.w = __builtin_fmaf(fmaxf(d, -150.0f), x, r.w);
    }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

template <int NT>
struct TopShared {
    float wave_m[NT / 64], wave_s[NT / 64], wave_w[NT / 64];
    alignas(16) unsigned group[kTopGroups];
    int reach[kTopGroups];
    unsigned long long list[kTopList];
    unsigned long long top[32];
    unsigned long long wave_key[NT / 64];
    unsigned bound;
    int reach_n, list_n;
};

// What a row (or a part of one) comes to.
__device__ __forceinline__ void write_row(const TokenRows& p, int64_t row, const Running& r, float given, bool has_token, int lane) {
    const bool none = r.m == kLowest && r.s == 0.0f;               // every token ruled out
    const bool bad = !(r.s < 3.402823466e+38f);                    // NaN or +inf in the row
    const float nan = __uint_as_float(0x7FC00000u);
    const float log_s = none ? 0.0f : logf(r.s);
    if (lane == 0) {
        if (p.logprob) p.logprob[row] = !has_token ? 0.0f : bad ? nan : (given - r.m) - log_s;
        if (p.entropy) p.entropy[row] = bad ? nan : none ? 0.0f : log_s - r.w / r.s;
    }
}
__device__ __forceinline__ void write_top(const TokenRows& p, int64_t row, const Running& r, int i, unsigned long long key) {
    const bool none = r.m == kLowest && r.s == 0.0f;
    const bool bad = !(r.s < 3.402823466e+38f);
    const float log_s = none ? 0.0f : logf(r.s);
    p.top_ids[row * p.k + i] = index_of(key);
    p.top_logprobs[row * p.k + i] = bad ? __uint_as_float(0x7FC00000u) : (value_of((unsigned)(key >> 32)) - r.m) - log_s;
}

// NT lanes per row (or part of a row), U 16-byte pieces a lane requested at once.
template <Elem T, int NT, int U>
__global__ __launch_bounds__(NT) void token_rows_kernel(TokenRows p) {
    constexpr int VEC = kVec<T>;
    constexpr int GW = NT / kTopGroups;                            // lanes of a group
    __shared__ TopShared<NT> sh;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = p.parts == 1 ? (int64_t)blockIdx.x : (int64_t)(blockIdx.x / (unsigned)p.parts);
    const int part = p.parts == 1 ? 0 : (int)(blockIdx.x % (unsigned)p.parts);
    const elem_t<T>* whole = static_cast<const elem_t<T>*>(p.logits) + row * p.ld;
    const int first = part * p.part_len;
    const int n = p.V - first < p.part_len ? p.V - first : p.part_len;
    const elem_t<T>* x = whole + first;

    int token = -1;
    float given = 0.0f;
    if (p.parts == 1 && p.tokens != nullptr) {
        token = p.tokens[row];
        if (token < 0 || token >= p.V) token = -1;
        if (token >= 0) given = elem_to_float<T>(whole[token]);
    }

    // pieces at 16-byte addresses; what lies before and behind them, at most VEC - 1 logits each, one lane each
    int head = (int)((16u - ((unsigned)(uintptr_t)x & 15u)) & 15u) / (int)sizeof(elem_t<T>);
    head = head < n ? head : n;
    const int body = (n - head) / VEC, rest = n - head - body * VEC;
    const elem_t<T>* xb = x + head;
    int edge = -1;                                                 // this lane's single logit
    if (tid < head) edge = tid;
    else if (tid >= VEC && tid - VEC < rest) edge = head + body * VEC + tid - VEC;
    Running r;
    float edge_v = 0.0f;
    if (edge >= 0) edge_v = elem_to_float<T>(x[edge]);

    int i0 = 0;
    for (; i0 + NT * U <= body; i0 += NT * U) {
        u32x4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = load_piece<T>(xb + (int64_t)(i0 + u * NT + tid) * VEC);
        float v[U * VEC];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[u * VEC + e] = piece_elem<T>(raw[u], e);
        add_logits(r, v);
    }
    for (; i0 + tid < body; i0 += NT) {
        const u32x4 raw = load_piece<T>(xb + (int64_t)(i0 + tid) * VEC);
        float v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = piece_elem<T>(raw, e);
        add_logits(r, v);
    }
    if (edge >= 0) {
        const float v[1] = {edge_v};
        add_logits(r, v);
    }

    // the row's maximum and sums
    const float mine = r.m;
    {
        const unsigned wm = wave_umax32(order_of(r.m));
        if (lane == 0) sh.wave_m[wave] = value_of(wm);
        if (tid == 0) sh.reach_n = sh.list_n = 0;
        if constexpr (GW == 1) {
            sh.group[tid] = order_of(mine);
        } else {
            float g = mine;
#pragma unroll
            for (int o = 1; o < GW; o <<= 1) g = fmaxf(g, __shfl_xor(g, o));
            if (tid % GW == 0) sh.group[tid / GW] = order_of(g);
        }
    }
    __syncthreads();
    float top = sh.wave_m[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) top = fmaxf(top, sh.wave_m[w]);
    raise(r, top);
    r.s = wave_sum(r.s);
    r.w = wave_sum(r.w);
    if (lane == 0) {
        sh.wave_s[wave] = r.s;
        sh.wave_w[wave] = r.w;
    }
    if (p.k > 0 && tid < kTopGroups) {
        const unsigned me = sh.group[tid];
        int ahead = 0;
        for (int j = 0; j < kTopGroups; j += 4) {
            const u32x4 o = *reinterpret_cast<const u32x4*>(&sh.group[j]);
#pragma unroll
            for (int e = 0; e < 4; ++e) ahead += o[e] > me || (o[e] == me && j + e < tid) ? 1 : 0;
        }
        if (ahead == p.k - 1) sh.bound = me;
    }
    __syncthreads();
    r.s = sh.wave_s[0];
    r.w = sh.wave_w[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) {
        r.s += sh.wave_s[w];
        r.w += sh.wave_w[w];
    }
    if (p.parts == 1) {
        write_row(p, row, r, given, token >= 0, tid);
    } else if (tid == 0) {
        float* to = p.sums + ((int64_t)row * p.parts + part) * 4;
        to[0] = r.m;
        to[1] = r.s;
        to[2] = r.w;
    }
    if (p.k == 0) return;

    const unsigned bound = sh.bound;
    const bool odd = !(r.s < 3.402823466e+38f);                    // NaN or +inf: the maxima do not show them all
    const int want = p.k < n ? p.k : n;
    if (tid < kTopGroups && sh.group[tid] >= bound) sh.reach[atomicAdd(&sh.reach_n, 1)] = tid;
    __syncthreads();
    auto offer = [&](float v, int index) {
        if (order_of(v) >= bound) {
            const int at = atomicAdd(&sh.list_n, 1);
            if (at < kTopList) sh.list[at] = key_of(v, first + index);
        }
    };
    if (!odd) {
        if (edge >= 0) offer(edge_v, edge);
        const int reach_n = sh.reach_n;
        for (int a = wave; a < reach_n; a += NT / 64) {
            const int t0 = sh.reach[a] * GW + lane % GW;
            for (int i = t0 + (lane / GW) * NT; i < body; i += (64 / GW) * NT) {
                const u32x4 raw = load_piece<T>(xb + (int64_t)i * VEC);
#pragma unroll
                for (int e = 0; e < VEC; ++e) offer(piece_elem<T>(raw, e), head + i * VEC + e);
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
    } else {
        for (int i = tid; i < got; i += NT) {
            const unsigned long long key = sh.list[i];
            int ahead = 0;
            for (int j = 0; j < got; ++j) ahead += sh.list[j] > key ? 1 : 0;
            if (ahead < want) sh.top[ahead] = key;
        }
        // fewer finite logits than alternatives: then all others are -inf, and the first of them follow
        for (int j0 = 0; got < want && j0 < n; j0 += 64) {         // (every wave the same; wave 0 writes)
            const float v = j0 + lane < n ? elem_to_float<T>(x[j0 + lane]) : 0.0f;
            const bool out = j0 + lane < n && v == -__builtin_inff();
            const unsigned long long mask = __ballot(out);
            const int at = got + (int)__popcll(mask & ((1ull << lane) - 1ull));
            if (wave == 0 && out && at < want) sh.top[at] = key_of(v, first + j0 + lane);
            got += (int)__popcll(mask);
        }
        __syncthreads();
    }
    if (tid < p.k) {
        const unsigned long long key = tid < want ? sh.top[tid] : 0ull;   // (a part shorter than k)
        if (p.parts == 1) write_top(p, row, r, tid, key);
        else p.keys[((int64_t)row * p.parts + part) * p.k + tid] = key;
    }
}

// The parts of a row joined by one wave, a lane per part: sums at the row's maximum, and the lists, each in order, merged.
template <Elem T>
__global__ __launch_bounds__(64) void token_join_kernel(TokenRows p) {
    const int lane = (int)threadIdx.x;
    const int64_t row = blockIdx.x;
    int token = -1;
    float given = 0.0f;
    if (p.tokens != nullptr) {
        token = p.tokens[row];
        if (token < 0 || token >= p.V) token = -1;
        if (token >= 0) given = elem_to_float<T>((static_cast<const elem_t<T>*>(p.logits) + row * p.ld)[token]);
    }
    Running r;
    const unsigned long long* keys = p.keys + ((int64_t)row * p.parts + lane) * p.k;
    unsigned long long next = 0;
    int used = 0;
    if (lane < p.parts) {
        const float* from = p.sums + ((int64_t)row * p.parts + lane) * 4;
        r.m = from[0];
        r.s = from[1];
        r.w = from[2];
        if (p.k > 0) next = keys[0];
    }
    raise(r, value_of(wave_umax32(order_of(r.m))));
    r.s = wave_sum(r.s);
    r.w = wave_sum(r.w);
    write_row(p, row, r, given, token >= 0, lane);
    for (int i = 0; i < p.k; ++i) {
        const unsigned hi = wave_umax32((unsigned)(next >> 32));
        const unsigned lo = wave_umax32((unsigned)(next >> 32) == hi ? (unsigned)next : 0u);
        const unsigned long long best = ((unsigned long long)hi << 32) | lo;
        if (next == best) {
            write_top(p, row, r, i, best);
            ++used;
            next = used < p.k ? keys[used] : 0ull;
        }
    }
}

struct TokenPlan {
    int parts, part_len;
    size_t keys_off, total;
};
static TokenPlan plan_token_rows(int64_t M, int64_t V, int k) {
    TokenPlan t{1, (int)V, 0, 0};
    int64_t parts = 1;
    if (M < compute_units()) {
        parts = compute_units() / (M > 0 ? M : 1);
        const int64_t most = V / 16384;
        parts = parts < most ? parts : most;
        parts = parts < 64 ? parts : 64;
        if (parts < 1) parts = 1;
    }
    if (parts > 1) {
        t.part_len = (int)round_up(ceil_div(V, parts), 64);
        t.parts = (int)ceil_div(V, t.part_len);
    }
    if (t.parts > 1) {
        t.keys_off = (size_t)round_up(M * t.parts * 16, 256);
        t.total = t.keys_off + (size_t)M * t.parts * k * 8;
    }
    return t;
}
size_t token_logprobs_workspace_bytes(int64_t M, int64_t V, int k) { return plan_token_rows(M, V, k).total; }

template <Elem T>
static hipError_t run_token_rows(const TokenRows& p, int64_t M, hipStream_t stream) {
    const int64_t groups = M * p.parts;
    if (groups > 0x7FFFFFFF) return hipErrorInvalidValue;
    const hipError_t e = groups < 2 * compute_units()
                             ? launch_kernel(0, token_rows_kernel<T, 1024, 2>, dim3((unsigned)groups), dim3(1024), 0, stream, p)
                             : launch_kernel(0, token_rows_kernel<T, 256, 4>, dim3((unsigned)groups), dim3(256), 0, stream, p);
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
