// Log probabilities of given tokens under rows of logits, the rows' entropy and their best alternatives, and the gradient:
//
//   m = max x over the allowed places, d_v = (x_v - m) scale log2(e), s = sum 2^d_v, t = sum 2^d_v d_v
//   logp_v = ln2 (d_v - log2 s),   entropy = ln2 (log2 s - t / s)
//   dlogits_v = scale (sum_{g: token_g = v} dlogp_g - p_v sum_g dlogp_g - dentropy p_v (logp_v + entropy))
//
// Differences from the maximum are formed before they are scaled, and m and log2 s are kept apart, so that rows of a type's
// lowest value keep their probabilities.  A place that is not allowed counts as -inf whatever it holds.  Sums are floats.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "policy.hpp"

namespace cpeval {

namespace {

constexpr int kThreads = 256;
constexpr float kNone = -INFINITY;
constexpr float kLift = 24.0f;
constexpr float kFar = -1000.0f;         // 2^kFar is 0: keeps 0 * -inf out of sums

struct Rows {
    int64_t rows;
    int32_t vocab;
    const void *logits;
    int64_t ld;
    float scale, unit;                   // unit: scale * log2(e)
    const uint64_t *allow;               // [rows][words], or null
    int32_t words;
};

struct Tokens {
    const void *at;
    int type;                            // bytes of one
    int64_t row_stride, stride;
    int32_t count;
    __device__ __forceinline__ int64_t get(int64_t row, int32_t g) const {
        const int64_t i = row * row_stride + g * stride;
        return type == 1 ? ((const uint8_t *)at)[i] : type == 4 ? ((const int32_t *)at)[i] : ((const int64_t *)at)[i];
    }
};

// one slice's sums, of the places it holds
struct Part {
    float m, s, t;
};

__device__ __forceinline__ Part joined(Part a, Part b, float unit) {
    const float m = fmaxf(a.m, b.m);
    if (m == kNone) return {m, a.s + b.s, a.t + b.t};
    const float da = fmaxf((a.m - m) * unit, kFar), db = fmaxf((b.m - m) * unit, kFar);
    const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
    return {m, fa * a.s + fb * b.s, fa * fmaf(a.s, da, a.t) + fb * fmaf(b.s, db, b.t)};
}

// a row with nothing allowed (and no NaN, which is not the same)
__device__ __forceinline__ bool is_empty(Part a) { return a.m == kNone && a.s == 0.0f; }
__device__ __forceinline__ float base_of(Part a) { return a.m == kNone ? 0.0f : a.m; }
__device__ __forceinline__ float log2_of(Part a) { return is_empty(a) ? 0.0f : __builtin_amdgcn_logf(a.s); }

// Larger logits first, ties by the lower place; 0: not an alternative.  (NaN counts as the largest, as in torch's orders.)
__device__ __forceinline__ uint64_t rank_key(float x, int32_t v) {
    if (x == kNone) return 0;
    uint32_t b = __float_as_uint(x + 0.0f);
    b = b & 0x80000000u ? ~b : b | 0x80000000u;
    return (uint64_t)b << 32 | (0xffffffffu - (uint32_t)v);
}
__device__ __forceinline__ int32_t key_place(uint64_t key) { return (int32_t)(0xffffffffu - (uint32_t)key); }
__device__ __forceinline__ float key_value(uint64_t key) {
    const uint32_t b = (uint32_t)(key >> 32);
    return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}

// which of the places from v on may be taken, the lowest bit first: as many as v's word still holds.  (The word is read in
// every case that has a mask, so that what depends on it is a choice between two values: hipcc has compiled a read behind
// a condition on both the mask's presence and a place's bit into code that lost the place's value.)
__device__ __forceinline__ uint64_t allowed_from(const Rows &r, int64_t row, int32_t v) {
    uint64_t bits = ~0ull;
    if (r.allow) bits = r.allow[row * r.words + (v >> 6)] >> (v & 63);
    return bits;
}

// log2 of the probability at a place, with the row's m and log2 s
__device__ __forceinline__ float log2_p(float x, float m, float l2s, float unit) { return x == kNone ? kNone : (x - m) * unit - l2s; }

// its natural logarithm (in these units the difference of two of a type's values fits the type)
__device__ __forceinline__ float log_p(const Rows &r, float x, float m, float l2s) {
    return x == kNone ? kNone : fmaf(x - m, r.scale, -kLn2 * l2s);
}

template <typename T>
__device__ __forceinline__ float logit(const Rows &r, int64_t row, int32_t v) {
    const float x = (float)((const T *)r.logits)[row * r.ld + v];
    return allowed_from(r, row, v) & 1 ? x : kNone;
}

__device__ __forceinline__ uint64_t wave_most(uint64_t v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const uint64_t o = __shfl_xor((unsigned long long)v, off);
        v = o > v ? o : v;
    }
    return v;
}

struct Results {
    float *logp, *entropy, *stats, *top_logp;
    int32_t *top_idx, top, *status;
};

// what is written of a row once its sums are known, by a workgroup: stats, entropy, tokens
template <typename T>
__device__ void write_row(const Rows &r, const Tokens &tok, const Results &out, int64_t row, Part all) {
    const float m = base_of(all), l2s = log2_of(all);
    const float entropy = is_empty(all) ? 0.0f : kLn2 * (l2s - all.t / all.s);
    if (threadIdx.x == 0) {
        out.entropy[row] = entropy;
        out.stats[3 * row] = m;
        out.stats[3 * row + 1] = l2s;
        out.stats[3 * row + 2] = entropy;
    }
    for (int32_t g = threadIdx.x; g < tok.count; g += blockDim.x) {
        const int64_t v = tok.get(row, g);
        float lp = 0.0f;
        if (v >= r.vocab) atomicOr(out.status, CP_STATUS_BAD_TOKEN);
        else if (v >= 0) lp = log_p(r, logit<T>(r, row, (int32_t)v), m, l2s);
        out.logp[row * tok.count + g] = lp;
    }
}

__device__ void write_top(const Rows &r, const Results &out, int64_t row, int i, uint64_t key, float m, float l2s) {
    out.top_idx[row * out.top + i] = key ? key_place(key) : -1;
    out.top_logp[row * out.top + i] = key ? log_p(r, key_value(key), m, l2s) : kNone;
}

// One slice of one row a workgroup, held in registers.  ONE: the slice is the whole row, and everything is written here;
// else its sums and its best places go to the workspace.
template <typename T, int V, int NV>
__global__ __launch_bounds__(kThreads) void slice_kernel(Rows r, Tokens tok, Results out, int32_t slices, Part *parts, uint64_t *best) {
    __shared__ float lds_m[4], lds_s[4], lds_t[4];
    __shared__ uint64_t lds_key[2][4];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t row = blockIdx.x / slices;
    const int32_t slice = blockIdx.x % slices, v0 = slice * (kThreads * V * NV);
    const T *from = (const T *)r.logits + row * r.ld;
    Pack<T, V> x[NV];
    float m = kNone;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int32_t v = v0 + (i * kThreads + threadIdx.x) * V;
        if (v < r.vocab) {
            x[i] = load_pack<T, V>(from + v);
            const uint64_t bits = allowed_from(r, row, v);
#pragma unroll
            for (int k = 0; k < V; k++) x[i].v[k] = bits >> k & 1 ? x[i].v[k] : (T)kNone;
        } else {
#pragma unroll
            for (int k = 0; k < V; k++) x[i].v[k] = (T)kNone;
        }
#pragma unroll
        for (int k = 0; k < V; k++) m = fmaxf(m, (float)x[i].v[k]);
    }
    m = wave_max(m);
    if (lane == 0) lds_m[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(lds_m[0], lds_m[1]), fmaxf(lds_m[2], lds_m[3]));
    float s = 0.0f, t = 0.0f;
    const float base = m == kNone ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
        for (int k = 0; k < V; k++) {
            const float d = ((float)x[i].v[k] - base) * r.unit, e = __builtin_amdgcn_exp2f(d);
            s += e;
            t = fmaf(e, fmaxf(d, kFar), t);
        }
    s = wave_sum(s);
    t = wave_sum(t);
    if (lane == 0) lds_s[wave] = s, lds_t[wave] = t;
    __syncthreads();
    const Part all = {m, (lds_s[0] + lds_s[1]) + (lds_s[2] + lds_s[3]), (lds_t[0] + lds_t[1]) + (lds_t[2] + lds_t[3])};
    if (slices == 1) write_row<T>(r, tok, out, row, all);
    else if (threadIdx.x == 0) parts[blockIdx.x] = all;

    uint64_t last = ~0ull;
    for (int q = 0; q < out.top; q++) {
        uint64_t key = 0;
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int k = 0; k < V; k++) {
                const uint64_t one = rank_key((float)x[i].v[k], v0 + (int32_t)((i * kThreads + threadIdx.x) * V) + k);
                key = one < last && one > key ? one : key;
            }
        key = wave_most(key);
        if (lane == 0) lds_key[q & 1][wave] = key;
        __syncthreads();
        for (int w = 0; w < 4; w++) key = lds_key[q & 1][w] > key ? lds_key[q & 1][w] : key;
        if (threadIdx.x == 0) {
            if (slices == 1) write_top(r, out, row, q, key, base, log2_of(all));
            else best[(int64_t)blockIdx.x * out.top + q] = key;
        }
        last = key;
    }
}

// a row's slices joined, in their order
template <typename T>
__global__ __launch_bounds__(kWave) void join_kernel(Rows r, Tokens tok, Results out, int32_t slices, const Part *parts, const uint64_t *best) {
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x;
    Part all = {kNone, 0.0f, 0.0f};
    for (int32_t i = lane; i < slices; i += kWave) all = joined(all, parts[row * slices + i], r.unit);
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const Part o = {__shfl_xor(all.m, off), __shfl_xor(all.s, off), __shfl_xor(all.t, off)};
        all = lane & off ? joined(o, all, r.unit) : joined(all, o, r.unit);
    }
    write_row<T>(r, tok, out, row, all);
    const float m = base_of(all), l2s = log2_of(all);
    uint64_t last = ~0ull;
    for (int q = 0; q < out.top; q++) {
        uint64_t key = 0;
        for (int64_t i = lane; i < (int64_t)slices * out.top; i += kWave) {
            const uint64_t one = best[row * slices * out.top + i];
            key = one < last && one > key ? one : key;
        }
        key = wave_most(key);
        if (lane == 0) write_top(r, out, row, q, key, m, l2s);
        last = key;
    }
}

struct Grads {
    const float *dlogp;
    int64_t row_stride, stride;
    const float *dentropy;
    int64_t de_stride;
};

// One row a workgroup: the softmax's part of every place, then what the tokens add at theirs.  A token's place is written
// by its first holder in the row, whole.
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void gradient_kernel(Rows r, Tokens tok, const float *stats, Grads d, float scale, T *out, int64_t ldo) {
    __shared__ float lds[4];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t row = blockIdx.x;
    const float m = stats[3 * row], l2s = stats[3 * row + 1], entropy = stats[3 * row + 2];
    const float de = d.dentropy ? d.dentropy[row * d.de_stride] : 0.0f;
    auto given = [&](int32_t g) {        // what token g's log probability passes on, and where
        const int64_t v = tok.get(row, g);
        const bool fine = v >= 0 && v < r.vocab && logit<T>(r, row, (int32_t)v) != kNone;
        return fine ? d.dlogp[row * d.row_stride + g * d.stride] : 0.0f;
    };
    float sum = 0.0f;
    for (int32_t g = threadIdx.x; g < tok.count; g += kThreads) sum += given(g);
    sum = wave_sum(sum);
    if (lane == 0) lds[wave] = sum;
    __syncthreads();
    sum = (lds[0] + lds[1]) + (lds[2] + lds[3]);
    // p (-sum - de (logp + entropy)) = p (flat + slope log2 p), with p lifted by 2^kLift: the hardware's exp gives 0 for what
    // lies below the normal numbers, its product with the rest need not
    const float slope = -de * kLn2, flat = -sum - de * entropy - kLift * slope + 0.0f * l2s;
    const float lift = exp2f(kLift), down = scale / lift, low = l2s - kLift;
    auto at = [&](float x, float hits) {
        const float l = log2_p(x, m, low, r.unit), p = __builtin_amdgcn_exp2f(l);
        return down * fmaf(p, fmaf(fmaxf(l, kFar), slope, flat), hits * lift);
    };
    for (int64_t v = (int64_t)threadIdx.x * V; v < r.vocab; v += kThreads * V) {
        const Pack<T, V> x = load_pack<T, V>((const T *)r.logits + row * r.ld + v);
        const uint64_t bits = allowed_from(r, row, (int32_t)v);
        Pack<T, V> o;
#pragma unroll
        for (int k = 0; k < V; k++) o.v[k] = (T)at(bits >> k & 1 ? (float)x.v[k] : kNone, 0.0f);
        store_pack<T, V>(out + row * ldo + v, o);
    }
    __syncthreads();
    for (int32_t g = threadIdx.x; g < tok.count; g += kThreads) {
        const int64_t v = tok.get(row, g);
        if (v < 0 || v >= r.vocab) continue;
        const float x = logit<T>(r, row, (int32_t)v);
        if (x == kNone) continue;
        bool mine = true;
        for (int32_t o = 0; o < g && mine; o++) mine = tok.get(row, o) != v;
        if (!mine) continue;
        float hits = 0.0f;
        for (int32_t o = g; o < tok.count; o++)
            if (tok.get(row, o) == v) hits += d.dlogp[row * d.row_stride + o * d.stride];
        out[row * ldo + v] = (T)at(x, hits);
    }
}

__global__ void clear_status_kernel(int32_t *status) { *status = CP_STATUS_OK; }

// (sixteen bytes a lane where rows allow it)
template <typename T>
bool wide(int32_t vocab, std::initializer_list<const void *> at, std::initializer_list<int64_t> ld) {
    constexpr int v = 16 / sizeof(T);
    for (const void *p : at)
        if ((uintptr_t)p % 16) return false;
    for (int64_t l : ld)
        if (l % v) return false;
    return vocab % v == 0;
}

constexpr int kMostLoads = 8;
constexpr int32_t slice_places(int v, int nv) { return kThreads * v * nv; }

// loads a thread: as many as leave the chip two workgroups a compute unit, and no more than the row has
int loads_of(int64_t rows, int32_t vocab, int v) {
    int nv = 1;
    while (nv < kMostLoads && slice_places(v, nv) < vocab && rows * ((vocab + slice_places(v, 2 * nv) - 1) / slice_places(v, 2 * nv)) >= 512) nv *= 2;
    return nv;
}

int check_rows(int64_t rows, int32_t vocab, int type, int32_t given, int token_type) {
    if (!known_type(type) || (given > 0 && token_type != CP_TOKEN_U8 && token_type != CP_TOKEN_I32 && token_type != CP_TOKEN_I64)) return CP_ERR_ARG;
    if (rows < 0 || rows > INT32_MAX || vocab < 1 || vocab > CP_LOGPROBS_MAX_VOCAB || given < 0) return CP_ERR_SIZE;
    return CP_OK;
}

// workgroups of the finest slicing that a call of these sizes can take
int64_t most_slices(int64_t rows, int32_t vocab) {
    const int64_t v1 = (vocab + slice_places(1, loads_of(rows, vocab, 1)) - 1) / slice_places(1, loads_of(rows, vocab, 1));
    const int64_t v4 = (vocab + slice_places(4, loads_of(rows, vocab, 4)) - 1) / slice_places(4, loads_of(rows, vocab, 4));
    const int64_t v8 = (vocab + slice_places(8, loads_of(rows, vocab, 8)) - 1) / slice_places(8, loads_of(rows, vocab, 8));
    return rows * std::max(v1, std::max(v4, v8));
}

}  // namespace

}  // namespace cpeval

using namespace cpeval;

extern "C" {

int cp_token_logprobs_workspace_bytes(int64_t rows, int32_t vocab, int32_t top, size_t *out_bytes) {
    if (!out_bytes) return CP_ERR_NULL;
    if (rows < 0 || rows > INT32_MAX || vocab < 1 || vocab > CP_LOGPROBS_MAX_VOCAB || top < 0 || top > CP_LOGPROBS_MAX_TOP) return CP_ERR_SIZE;
    const int64_t n = most_slices(rows, vocab);
    *out_bytes = align_up(n * sizeof(Part)) + align_up(n * top * sizeof(uint64_t));
    return CP_OK;
}

int cp_token_logprobs(int64_t rows, int32_t vocab, int type, const void *logits, int64_t ld, float scale, const uint64_t *allow,
                      int32_t given, const void *tokens, int token_type, int64_t token_row_stride, int64_t token_stride, float *logp,
                      float *entropy, float *stats, int32_t top, float *top_logp, int32_t *top_idx, void *workspace,
                      size_t workspace_bytes, void *stream, int32_t *status_out) {
    int rc = check_rows(rows, vocab, type, given, token_type);
    if (rc) return rc;
    if (top < 0 || top > CP_LOGPROBS_MAX_TOP) return CP_ERR_SIZE;
    if (!(scale > 0.0f) || scale > 3.0e38f) return CP_ERR_ARG;
    if (!status_out) return CP_ERR_NULL;
    if (rows > 0 && (!logits || !entropy || !stats || (given && (!tokens || !logp)) || (top && (!top_logp || !top_idx)))) return CP_ERR_NULL;
    if (rows > 1 && ld < vocab) return CP_ERR_SIZE;
    size_t need = 0;
    cp_token_logprobs_workspace_bytes(rows, vocab, top, &need);
    if (need && !workspace) return CP_ERR_NULL;
    if ((uintptr_t)workspace % kPolicyAlign || workspace_bytes < need) return CP_ERR_WORKSPACE;
    const hipStream_t st = (hipStream_t)stream;
    hipLaunchKernelGGL(clear_status_kernel, dim3(1), dim3(1), 0, st, status_out);
    if (rows == 0) return launched();
    const Rows r{rows, vocab, logits, ld, scale, scale * kLog2e, allow, (vocab + 63) / 64};
    const Tokens tok{tokens, token_type, token_row_stride, token_stride, given};
    const Results out{logp, entropy, stats, top_logp, top_idx, top, status_out};
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        auto go = [&](auto v) {
            constexpr int V = decltype(v)::value;
            const int nv = loads_of(rows, vocab, V);
            const int32_t slices = (vocab + slice_places(V, nv) - 1) / slice_places(V, nv);
            if (rows * slices > INT32_MAX) return (int)CP_ERR_SIZE;
            Part *parts = (Part *)workspace;
            uint64_t *best = (uint64_t *)((char *)workspace + align_up((size_t)rows * slices * sizeof(Part)));
            auto run = [&](auto n) {
                constexpr int NV = decltype(n)::value;
                hipLaunchKernelGGL((slice_kernel<T, V, NV>), dim3((unsigned)(rows * slices)), dim3(kThreads), 0, st, r, tok, out, slices, parts, best);
            };
            if (nv == 1) run(std::integral_constant<int, 1>{});
            else if (nv == 2) run(std::integral_constant<int, 2>{});
            else if (nv == 4) run(std::integral_constant<int, 4>{});
            else run(std::integral_constant<int, 8>{});
            if (slices > 1) hipLaunchKernelGGL((join_kernel<T>), dim3((unsigned)rows), dim3(kWave), 0, st, r, tok, out, slices, parts, best);
            return launched();
        };
        constexpr int V = 16 / sizeof(T);
        if (wide<T>(vocab, {logits}, {ld})) return go(std::integral_constant<int, V>{});
        return go(std::integral_constant<int, 1>{});
    });
}

int cp_token_logprobs_backward(int64_t rows, int32_t vocab, int type, const void *logits, int64_t ld, float scale, const uint64_t *allow,
                               int32_t given, const void *tokens, int token_type, int64_t token_row_stride, int64_t token_stride,
                               const float *stats, const float *dlogp, int64_t dlogp_row_stride, int64_t dlogp_stride,
                               const float *dentropy, int64_t dentropy_stride, void *dlogits, int64_t ldd, void *stream) {
    int rc = check_rows(rows, vocab, type, given, token_type);
    if (rc) return rc;
    if (!(scale > 0.0f) || scale > 3.0e38f) return CP_ERR_ARG;
    if (rows > 0 && (!logits || !stats || !dlogits || (given && (!tokens || !dlogp)))) return CP_ERR_NULL;
    if (rows > 1 && (ld < vocab || ldd < vocab)) return CP_ERR_SIZE;
    if (rows == 0) return CP_OK;
    const Rows r{rows, vocab, logits, ld, scale, scale * kLog2e, allow, (vocab + 63) / 64};
    const Tokens tok{tokens, token_type, token_row_stride, token_stride, given};
    const Grads d{dlogp, dlogp_row_stride, dlogp_stride, dentropy, dentropy_stride};
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        auto go = [&](auto v) {
            constexpr int V = decltype(v)::value;
            hipLaunchKernelGGL((gradient_kernel<T, V>), dim3((unsigned)rows), dim3(kThreads), 0, (hipStream_t)stream, r, tok, stats, d, scale,
                               (T *)dlogits, ldd);
            return launched();
        };
        constexpr int V = 16 / sizeof(T);
        if (wide<T>(vocab, {logits, dlogits}, {ld, ldd})) return go(std::integral_constant<int, V>{});
        return go(std::integral_constant<int, 1>{});
    });
}

}  // extern "C"
