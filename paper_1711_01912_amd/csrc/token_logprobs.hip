// Log probabilities of given tokens under rows of logits, the rows' entropy and their best alternatives, and the gradient:
//
//   m = max x over the allowed places, d_v = (x_v - m) scale log2(e), s = sum 2^d_v, t = sum 2^d_v d_v
//   logp_v = ln2 (d_v - log2 s),   entropy = ln2 (log2 s - t / s)
//   dlogits_v = scale (sum_{g: token_g = v} dlogp_g - p_v sum_g dlogp_g - dentropy p_v (logp_v + entropy))
//
// Differences from the maximum are formed before they are scaled, and m and log2 s are kept apart, so that rows of a type's
// lowest value keep their probabilities.  A place that is not allowed counts as -inf whatever it holds.  Sums are floats, also
// those over a row's tokens: a gradient of 1,024 tokens a row is off by 1e-7 to 8e-7 of its size, as the tokens' weights cancel, one
// with these sums in 64 bits by 0.6e-7 to 1.5e-7.
//
// Bound by memory where rows are long: 8192 x 65536 bf16 take 208 us forward (5.1 TB/s, the rate of a copy) and 365 us backward
// (5.9 TB/s, some of it from the caches).  Rows of few places with many tokens: 200000 x 8 with 1024 tokens of a byte 265 us
// forward (3.8 TB/s read and written; 166 us where the tokens are still in the caches), 113 backward, where each token is a
// read and a write of a sum in LDS, and lanes whose tokens differ meet in the same banks: 64 % of the LDS's busy cycles.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <climits>

#include "policy.hpp"

namespace cpeval {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
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

// The larger of three, as one instruction (fmaxf makes each operand a quiet NaN first, by one of its own).  A quiet NaN is
// passed over, a signalling one makes the result a quiet NaN, which hides what was in front of it.
__device__ __forceinline__ float max_of(float a, float b, float c) {
    float m;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}

// sums over some of a row's places
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
__device__ __forceinline__ float entropy_of(Part a) { return is_empty(a) ? 0.0f : kLn2 * (log2_of(a) - a.t / a.s); }

// Larger logits first, ties by the lower place; 0: not an alternative (-inf, a NaN)
__device__ __forceinline__ uint32_t value_key(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t rank_key(float x, int32_t v) {
    return !(x > kNone) ? 0 : (uint64_t)value_key(x) << 32 | (0xffffffffu - (uint32_t)v);
}
__device__ __forceinline__ int32_t key_place(uint64_t key) { return (int32_t)(0xffffffffu - (uint32_t)key); }
__device__ __forceinline__ float key_value(uint64_t key) {
    const uint32_t b = (uint32_t)(key >> 32);
    return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
constexpr uint32_t kNoneKey = 0x007fffffu;       // value_key(-inf)

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

// maxima and sums over groups of L neighbouring lanes, in all of them
template <int L>
__device__ __forceinline__ uint64_t most(uint64_t v) {
#pragma unroll
    for (int off = L / 2; off > 0; off >>= 1) {
        const uint64_t o = __shfl_xor((unsigned long long)v, off);
        v = o > v ? o : v;
    }
    return v;
}
template <int L>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
    for (int off = L / 2; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}
template <int L>
__device__ __forceinline__ float group_add(float v) {
#pragma unroll
    for (int off = L / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

struct Results {
    float *logp, *entropy, *stats, *top_logp;
    int32_t *top_idx, top, *status;
    bool stream;             // logp goes past the caches
};

__device__ __forceinline__ void write_sums(const Results &out, int64_t row, Part all) {
    const float entropy = entropy_of(all);
    out.entropy[row] = entropy;
    out.stats[3 * row] = base_of(all);
    out.stats[3 * row + 1] = log2_of(all);
    out.stats[3 * row + 2] = entropy;
}

// a row's tokens, by a workgroup
template <typename T>
__device__ void write_tokens(const Rows &r, const Tokens &tok, const Results &out, int64_t row, Part all) {
    const float m = base_of(all), l2s = log2_of(all);
    for (int32_t g = threadIdx.x; g < tok.count; g += blockDim.x) {
        const int64_t v = tok.get(row, g);
        float lp = 0.0f;
        if (v >= r.vocab) atomicOr(out.status, CP_STATUS_BAD_TOKEN);
        else if (v >= 0) lp = log_p(r, logit<T>(r, row, (int32_t)v), m, l2s);
        out.logp[row * tok.count + g] = lp;
    }
}

__device__ void write_top(const Rows &r, const Results &out, int64_t row, int i, uint64_t key, Part all) {
    out.top_idx[row * out.top + i] = key ? key_place(key) : -1;
    out.top_logp[row * out.top + i] = key ? log_p(r, key_value(key), base_of(all), log2_of(all)) : kNone;
}

// ---- rows of many places ----
//
// A workgroup takes a slice of a row into registers: exact maximum first, then the sums, with no rescaling on the way, and
// the row is read once.  Rows are cut into as few slices as leave the chip enough workgroups; what they find is joined by a
// second launch.

// A slice's loads: NV vectors a thread.  The last vector of a row that is no multiple of V is the row's last V places, those
// of them that belong to another vector counting as not there.
template <typename T, int V, int NV>
struct Slice {
    Raw<T, V> x[NV];
    int32_t v0;

    __device__ __forceinline__ int32_t first(int i) const { return v0 + (i * kThreads + (int32_t)threadIdx.x) * V; }
    __device__ __forceinline__ int32_t place(const Rows &r, int i) const { return min(first(i), r.vocab - V); }

    __device__ __forceinline__ void load(const Rows &r, int64_t row, int32_t slice) {
        v0 = slice * (kThreads * V * NV);
        const T *from = (const T *)r.logits + row * r.ld;
#pragma unroll
        for (int i = 0; i < NV; i++) x[i].load(from + max(place(r, i), 0));
    }
    // which of a vector's places count, the lowest bit first
    __device__ __forceinline__ uint64_t counts(const Rows &r, int64_t row, int i) const {
        const int32_t v = first(i);
        const uint64_t own = v < r.vocab ? ~0ull << (v - place(r, i)) : 0;
        const uint64_t may = allowed_from(r, row, min(v, r.vocab - 1));
        return own & (may << (v < r.vocab ? v - place(r, i) : 0));
    }
    __device__ __forceinline__ void blank(const Rows &r, int64_t row) {
        // (all of the places of most slices count)
        if (!r.allow && v0 + kThreads * V * NV <= r.vocab) return;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const uint64_t bits = counts(r, row, i);
#pragma unroll
            for (int k = 0; k < V; k++) x[i].set_none(k, bits >> k & 1);
        }
    }
};

// A bound that at least `top` of a workgroup's value keys reach, and few more: `key` is the largest of each thread's.  Of each
// wavefront whose threads all have some, a share of `top` (together: `top`) reach the share-th largest of theirs, found bit
// by bit, and the lowest of these counts.  (A wavefront without any would leave no bound: 5250 rows of 1401 bf16, the 20 best
// of each, took 146 us so.)  `threads`: so many have some.
__device__ __forceinline__ uint32_t bound_of(uint32_t key, int top, int threads) {
    __shared__ uint32_t lds[kWaves];
    const int full = max(1, min(kWaves, threads / kWave)), share = (top + full - 1) / full;
    uint32_t bound = 0;
#pragma unroll
    for (int bit = 31; bit >= 0; bit--) {
        const uint32_t more = bound | 1u << bit;
        bound = __popcll(__ballot(key >= more)) >= share ? more : bound;
    }
    if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x / kWave] = bound;
    __syncthreads();
    bound = lds[0];
    for (int w = 1; w < full; w++) bound = min(bound, lds[w]);
    return max(bound, kNoneKey + 1);
}

// The best places of a slice.  `own`: the thread's largest logit.  Those at or above the bound are all that is put in order.
// Where too many are (ties), the best are taken one by one, from memory.
constexpr int kPool = 512;
template <typename T, int V, int NV, typename F>
__device__ __forceinline__ void slice_top(const Rows &r, int64_t row, Slice<T, V, NV> &in, float own, int top, F put) {
    __shared__ uint64_t lds_pool[kPool], lds_key[2][kWaves];
    __shared__ int lds_count;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const uint32_t key = own > kNone ? value_key(own) : 0;
    if (threadIdx.x == 0) lds_count = 0;
    const uint32_t bound = bound_of(key, top, (r.vocab - in.v0) / V);
    if (key >= bound) {
        const float low = key_value((uint64_t)bound << 32);
#pragma unroll
        for (int i = 0; i < NV; i++) {
            in.x[i].renew();
#pragma unroll
            for (int k = 0; k < V; k++) {
                if (!(in.x[i][k] >= low)) continue;
                const int at = atomicAdd(&lds_count, 1);
                if (at < kPool) lds_pool[at] = rank_key(in.x[i][k], in.place(r, i) + k);
            }
        }
    }
    __syncthreads();
    const int count = lds_count;
    if (count <= kPool) {
        for (int i = threadIdx.x; i < count; i += kThreads) {
            const uint64_t key = lds_pool[i];
            int rank = 0;
            for (int o = 0; o < count; o++) rank += lds_pool[o] > key;
            if (rank < top) put(rank, key);
        }
        for (int i = count + threadIdx.x; i < top; i += kThreads) put(i, 0);
        return;
    }
    uint64_t last = ~0ull;
    for (int q = 0; q < top; q++) {
        uint64_t key = 0;
        for (int32_t v = in.v0 + threadIdx.x; v < min(in.v0 + kThreads * V * NV, r.vocab); v += kThreads) {
            const uint64_t one = rank_key(logit<T>(r, row, v), v);
            key = one < last && one > key ? one : key;
        }
        key = most<kWave>(key);
        if (lane == 0) lds_key[q & 1][wave] = key;
        __syncthreads();
        for (int w = 0; w < kWaves; w++) key = lds_key[q & 1][w] > key ? lds_key[q & 1][w] : key;
        if (threadIdx.x == 0) put(q, key);
        last = key;
    }
}

// One slice of one row a workgroup.  One slice a row: everything is written here; else its sums and its best places go to the
// workspace.
template <typename T, int V, int NV, bool TOP>
__global__ __launch_bounds__(kThreads, 4) void slice_kernel(Rows r, Tokens tok, Results out, int32_t slices, Part *parts, uint64_t *best) {
    __shared__ float lds_m[kWaves], lds_s[kWaves], lds_t[kWaves];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const uint32_t number = group_number();
    const int64_t row = number / (uint32_t)slices;
    if (row >= r.rows) return;
    Slice<T, V, NV> in;
    in.load(r, row, (int32_t)(number - (uint32_t)row * (uint32_t)slices));
    in.blank(r, row);
    if (slices > 1 && number == 0 && threadIdx.x == 0) *out.status = CP_STATUS_OK;       // (tokens are looked at by the next launch)
    float m = kNone;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        in.x[i].renew();
#pragma unroll
        for (int k = 0; k < V; k += 2) m = max_of(m, in.x[i][k], in.x[i][k + 1]);
    }
    float own = m;
    m = wave_max(m);
    if (lane == 0) lds_m[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(lds_m[0], lds_m[1]), fmaxf(lds_m[2], lds_m[3]));
    float s[2] = {0.0f, 0.0f}, t[2] = {0.0f, 0.0f};
    const float base = m == kNone ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        in.x[i].renew();
#pragma unroll
        for (int k = 0; k < V; k++) {
            const float d = (in.x[i][k] - base) * r.unit, e = __builtin_amdgcn_exp2f(d);
            s[k & 1] += e;
            t[k & 1] = fmaf(e, fmaxf(d, kFar), t[k & 1]);
        }
    }
    s[0] = wave_sum(s[0] + s[1]);
    t[0] = wave_sum(t[0] + t[1]);
    if (lane == 0) lds_s[wave] = s[0], lds_t[wave] = t[0];
    __syncthreads();
    const Part all = {m, (lds_s[0] + lds_s[1]) + (lds_s[2] + lds_s[3]), (lds_t[0] + lds_t[1]) + (lds_t[2] + lds_t[3])};
    if (TOP && !(all.s == all.s)) {          // (with a NaN about, which is no alternative but may have hidden some)
        own = kNone;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            in.x[i].renew();
#pragma unroll
            for (int k = 0; k < V; k++) own = in.x[i][k] > own ? in.x[i][k] : own;
        }
    }
    if (slices == 1) {
        if (threadIdx.x == 0) write_sums(out, row, all);
        write_tokens<T>(r, tok, out, row, all);
        if constexpr (TOP) slice_top<T, V, NV>(r, row, in, own, out.top, [&](int i, uint64_t key) { write_top(r, out, row, i, key, all); });
    } else {
        if (threadIdx.x == 0) parts[number] = all;
        if constexpr (TOP) slice_top<T, V, NV>(r, row, in, own, out.top, [&](int i, uint64_t key) { best[(int64_t)number * out.top + i] = key; });
    }
}

// A row's slices joined, in their order, and the best of their best places.
template <typename T>
__global__ __launch_bounds__(kThreads) void join_kernel(Rows r, Tokens tok, Results out, int32_t slices, const Part *parts, const uint64_t *best) {
    __shared__ Part lds_part;
    __shared__ uint64_t lds_pool[kPool], lds_key[kWaves];
    __shared__ int lds_count;
    const int64_t row = group_number();
    if (row >= r.rows) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    if (wave == 0) {
        Part all = {kNone, 0.0f, 0.0f};
        for (int32_t i = lane; i < slices; i += kWave) all = joined(all, parts[row * slices + i], r.unit);
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const Part o = {__shfl_xor(all.m, off), __shfl_xor(all.s, off), __shfl_xor(all.t, off)};
            all = lane & off ? joined(o, all, r.unit) : joined(all, o, r.unit);
        }
        if (lane == 0) {
            lds_part = all;
            lds_count = 0;
            write_sums(out, row, all);
        }
    }
    const int64_t count = (int64_t)slices * out.top;
    const uint64_t *keys = best + row * count;
    uint32_t bound = 0;
    if (out.top) {
        for (int64_t i = threadIdx.x; i < count; i += kThreads) bound = max(bound, (uint32_t)(keys[i] >> 32));
        bound = bound_of(bound, out.top, (int)min(count, (int64_t)kThreads));
    }
    __syncthreads();
    const Part all = lds_part;
    write_tokens<T>(r, tok, out, row, all);
    if (!out.top) return;
    for (int64_t i = threadIdx.x; i < count; i += kThreads) {
        const uint64_t key = keys[i];
        if ((uint32_t)(key >> 32) < bound) continue;
        const int at = atomicAdd(&lds_count, 1);
        if (at < kPool) lds_pool[at] = key;
    }
    __syncthreads();
    const int found = lds_count;
    if (found <= kPool) {
        for (int i = threadIdx.x; i < found; i += kThreads) {
            int rank = 0;
            for (int o = 0; o < found; o++) rank += lds_pool[o] > lds_pool[i];
            if (rank < out.top) write_top(r, out, row, rank, lds_pool[i], all);
        }
        for (int i = found + threadIdx.x; i < out.top; i += kThreads) write_top(r, out, row, i, 0, all);
        return;
    }
    uint64_t last = ~0ull;
    for (int q = 0; q < out.top; q++) {
        uint64_t key = 0;
        for (int64_t i = threadIdx.x; i < count; i += kThreads) key = keys[i] < last && keys[i] > key ? keys[i] : key;
        key = most<kWave>(key);
        __syncthreads();
        if (lane == 0) lds_key[wave] = key;
        __syncthreads();
        for (int w = 0; w < kWaves; w++) key = lds_key[w] > key ? lds_key[w] : key;
        if (threadIdx.x == 0) write_top(r, out, row, q, key, all);
        last = key;
    }
}

struct Grads {
    const float *dlogp;
    int64_t row_stride, stride;
    const float *dentropy;
    int64_t de_stride;
    __device__ __forceinline__ float get(int64_t row, int32_t g) const { return dlogp[row * row_stride + g * stride]; }
};

// A row's gradient, place by place: scale (hits + p (-sum - de (logp + entropy))) = scale (hits + p (flat + slope log2 p)).
// p is lifted by 2^kLift: the hardware's exp gives 0 for what lies below the normal numbers, its product with the rest need
// not.  A place without a probability gets 0 itself, since what its row passes on may be infinite, and 0 times that a NaN.
struct Slope {
    float m, low, unit, slope, flat, down;
    __device__ __forceinline__ Slope(const Rows &r, const float *stats, float de, float sum) {
        const float l2s = stats[1];
        m = stats[0];
        unit = r.unit;
        low = l2s - kLift;
        slope = -de * kLn2;
        flat = -sum - de * stats[2] - kLift * slope + 0.0f * l2s;        // (NaN where the row's sums are)
        down = r.scale / exp2f(kLift);
    }
    __device__ __forceinline__ float at(float x, float hits) const {
        const float l = log2_p(x, m, low, unit), p = __builtin_amdgcn_exp2f(l);
        const float all = down * fmaf(p, fmaf(fmaxf(l, kFar), slope, flat), hits * exp2f(kLift));
        return x == kNone ? 0.0f : all;
    }
};

// One slice of one row a workgroup: the softmax's part of every place, then what the tokens add at theirs.  A token's place
// is written by its first holder in the row, whole.  No place is written by two workgroups: the last vector of a row, moved
// back to end with it, may begin in the slice before, whose workgroup adds the tokens there.
template <typename T, int V, int NV>
__global__ __launch_bounds__(kThreads) void gradient_kernel(Rows r, Tokens tok, const float *stats, Grads d, T *out, int64_t ldo, int32_t slices, bool stream) {
    __shared__ float lds[kWaves];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const uint32_t number = group_number();
    const int64_t row = number / (uint32_t)slices;
    if (row >= r.rows) return;
    Slice<T, V, NV> in;
    in.load(r, row, (int32_t)(number - (uint32_t)row * (uint32_t)slices));
    auto given = [&](int32_t g) {        // what token g's log probability passes on
        const int64_t v = tok.get(row, g);
        const bool fine = v >= 0 && v < r.vocab && logit<T>(r, row, (int32_t)v) != kNone;
        return fine ? d.get(row, g) : 0.0f;
    };
    float sum = 0.0f;
    if (tok.count == 1) {
        sum = given(0);
    } else if (tok.count > 1) {
        for (int32_t g = threadIdx.x; g < tok.count; g += kThreads) sum += given(g);
        sum = wave_sum(sum);
        if (lane == 0) lds[wave] = sum;
        __syncthreads();
        sum = (lds[0] + lds[1]) + (lds[2] + lds[3]);
    }
    const Slope slope(r, stats + 3 * row, d.dentropy ? d.dentropy[row * d.de_stride] : 0.0f, sum);
    // (the places that do not count get what their owner gives them)
    const int64_t only = tok.count == 1 ? tok.get(row, 0) : -1;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int32_t v = in.place(r, i);
        if (in.first(i) >= r.vocab) continue;
        uint64_t may = ~0ull;
        if (r.allow) {
            may = r.allow[row * r.words + (v >> 6)] >> (v & 63);
            if ((v & 63) + V > 64) may |= r.allow[row * r.words + (v >> 6) + 1] << (64 - (v & 63));
        }
        Pack<T, V> o;
#pragma unroll
        for (int k = 0; k < V; k++) o.v[k] = (T)slope.at(may >> k & 1 ? in.x[i][k] : kNone, 0.0f);
        const int64_t to = only - v;
        if (to >= 0 && to < V) {
#pragma unroll
            for (int k = 0; k < V; k++)
                if (to == k && (may >> k & 1) && in.x[i][k] != kNone) o.v[k] = (T)slope.at(in.x[i][k], sum);
        }
        T *to_v = out + row * ldo + v;
        if (i == 0 && v < in.v0) {           // (a slice of fewer than V places: its first vector is the row's last)
#pragma unroll
            for (int k = 0; k < V; k++)
                if (v + k >= in.v0) to_v[k] = o.v[k];
        } else {
            store_pack<T, V>(to_v, o, stream);
        }
    }
    if (tok.count < 2) return;
    __syncthreads();
    const int32_t low = in.v0, high = min(in.v0 + kThreads * V * NV, r.vocab);
    for (int32_t g = threadIdx.x; g < tok.count; g += kThreads) {
        const int64_t v = tok.get(row, g);
        if (v < low || v >= high) continue;
        const float x = logit<T>(r, row, (int32_t)v);
        if (x == kNone) continue;
        bool mine = true;
        for (int32_t o = 0; o < g && mine; o++) mine = tok.get(row, o) != v;
        if (!mine) continue;
        float hits = 0.0f;
        for (int32_t o = g; o < tok.count; o++)
            if (tok.get(row, o) == v) hits += d.get(row, o);
        out[row * ldo + v] = (T)slope.at(x, hits);
    }
}

// ---- rows of few places, such as devices ----
//
// Some neighbouring lanes a row, kEach of its places a lane, several rows a wavefront, so that what is done once a row is done
// for many at once.  (A place a lane, a wavefront took 362 us for a million rows of 64 bf16 logits and four tokens, most of it
// for moving sums from lane to lane.)  The row's log probabilities are a table in LDS for its tokens, of which there may be as
// many as partitions were drawn.

// Four tokens from g on, side by side or `stride` apart; behind the last, the last again (whose results go nowhere, and whose
// weights are 0)
template <typename I>
struct Four {
    Pack<I, 4> v;
    __device__ __forceinline__ void load(const Tokens &tok, int64_t row, int32_t g) {
        const I *at = (const I *)tok.at + row * tok.row_stride;
        if (tok.stride == 1 && g + 4 <= tok.count) v = load_pack<I, 4>(at + g);
        else
#pragma unroll
            for (int j = 0; j < 4; j++) v.v[j] = at[(int64_t)min(g + j, tok.count - 1) * tok.stride];
    }
    // the place of the j-th, or -1 for one to be ignored; `bad`: it lies behind the last place
    __device__ __forceinline__ int place(int j, int32_t vocab, bool &bad) const {
        if constexpr (sizeof(I) == 8) {
            bad |= v.v[j] >= vocab;
            return v.v[j] >= 0 && v.v[j] < vocab ? (int)v.v[j] : -1;
        } else {
            bad |= (int32_t)v.v[j] >= vocab;
            return (uint32_t)v.v[j] < (uint32_t)vocab ? (int)v.v[j] : -1;
        }
    }
};
constexpr int kAhead = 4;                // fours a lane loads before it looks at them

constexpr int kEach = 8;

// The places of a row that a lane has: kEach from `at` on, the last of them the row's last (of shorter rows: all), so that
// some may be its neighbour's, which counts them.
struct Few {
    int32_t at;
    uint32_t here, mine;                 // bit e: at + e is a place of the row; and it is counted by this lane
    __device__ __forceinline__ Few(int32_t vocab, int part) {
        const int32_t first = part * kEach, behind = first < vocab ? min(vocab - first, kEach) : 0;
        at = max(min(first, vocab - kEach), 0);
        here = (1u << min(vocab, kEach)) - 1;
        mine = ((1u << behind) - 1) << (behind ? first - at : 0);
    }
    // their logits, -inf where not allowed
    template <typename T>
    __device__ __forceinline__ void load(float (&x)[kEach], const Rows &r, int64_t row) const {
        const T *from = (const T *)r.logits + row * r.ld + at;
        if (r.vocab >= kEach) {
            Raw<T, kEach> raw;
            raw.load(from);
#pragma unroll
            for (int e = 0; e < kEach; e++) x[e] = raw[e];
        } else {
#pragma unroll
            for (int e = 0; e < kEach; e++) x[e] = (float)from[min(e, r.vocab - 1)];
        }
        if (r.allow) {
            const uint64_t *word = r.allow + row * r.words + (at >> 6);
            uint64_t may = word[0] >> (at & 63);
            if ((at & 63) + kEach > 64) may |= word[1] << (64 - (at & 63));
#pragma unroll
            for (int e = 0; e < kEach; e++) x[e] = may >> e & 1 ? x[e] : kNone;
        }
    }
};

// what a wavefront's lanes have written to LDS is there for all of them
__device__ __forceinline__ void lds_ready() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// `lanes` (a multiple of S) lanes a row: S neighbours have its places, and where lanes are more than S, others the same again;
// for its tokens each of them is another.
template <typename T, typename I, int S>
__global__ __launch_bounds__(kThreads, 4) void few_kernel(Rows r, Tokens tok, Results out, int lanes) {
    constexpr int kPitch = S * kEach + 1;
    __shared__ float lds[kWaves][kWave / S * kPitch];
    const int lane = threadIdx.x & (kWave - 1), here = lane & (lanes - 1), group = lane / lanes;
    float *table = lds[threadIdx.x / kWave] + group * kPitch;
    const Few few(r.vocab, lane & (S - 1));
    bool bad = false;
    const int side = kWave / lanes;
    const int64_t step = (int64_t)gridDim.x * kWaves * side;
    int64_t row0 = ((int64_t)blockIdx.x * kWaves + threadIdx.x / kWave) * side;
    float soon[kEach];
    few.load<T>(soon, r, min(row0 + group, r.rows - 1));
    for (; row0 < r.rows; row0 += step) {
        const int64_t row = min(row0 + group, r.rows - 1);
        const bool live = row0 + group < r.rows;
        // what memory has to give is asked for first: this row's tokens, the next row's logits
        Four<I> four[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; a++)
            if ((here + a * lanes) * 4 < tok.count) four[a].load(tok, row, (here + a * lanes) * 4);
        float x[kEach], m = kNone;
#pragma unroll
        for (int e = 0; e < kEach; e++) {
            x[e] = few.mine >> e & 1 ? soon[e] : kNone;
            m = fmaxf(m, x[e]);
        }
        few.load<T>(soon, r, min(row0 + step + group, r.rows - 1));
        Part all = {group_max<S>(m), 0.0f, 0.0f};
        const float base = base_of(all);
#pragma unroll
        for (int e = 0; e < kEach; e++) {
            const float d = (x[e] - base) * r.unit, p = __builtin_amdgcn_exp2f(d);
            all.s += p;
            all.t = fmaf(p, fmaxf(d, kFar), all.t);
        }
        all.s = group_add<S>(all.s);
        all.t = group_add<S>(all.t);
        const float l2s = log2_of(all);
        if (live && here == 0) write_sums(out, row, all);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int e = 0; e < kEach; e++)
            if (few.mine >> e & 1) table[few.at + e] = log_p(r, x[e], base, l2s);
        lds_ready();
        for (int32_t g0 = here * 4; g0 < tok.count; g0 += kAhead * lanes * 4) {
            if (g0 > here * 4) {
#pragma unroll
                for (int a = 0; a < kAhead; a++)
                    if (g0 + a * lanes * 4 < tok.count) four[a].load(tok, row, g0 + a * lanes * 4);
            }
#pragma unroll
            for (int a = 0; a < kAhead; a++) {
                const int32_t g = g0 + a * lanes * 4;
                if (g >= tok.count || !live) continue;
                Pack<float, 4> lp;
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const int v = four[a].place(j, r.vocab, bad);
                    lp.v[j] = table[max(v, 0)];
                    lp.v[j] = v >= 0 ? lp.v[j] : 0.0f;
                }
                float *to = out.logp + row * tok.count + g;
                if (g + 4 <= tok.count) store_pack<float, 4>(to, lp, out.stream);
                else
#pragma unroll
                    for (int j = 0; j < 4; j++)
                        if (g + j < tok.count) to[j] = lp.v[j];
            }
        }
        uint64_t last = ~0ull;
        for (int q = 0; q < out.top; q++) {
            uint64_t key = 0;
#pragma unroll
            for (int e = 0; e < kEach; e++) {
                const uint64_t one = rank_key(x[e], few.at + e);
                key = one < last && one > key ? one : key;
            }
            key = most<S>(key);
            if (live && here == 0) write_top(r, out, row, q, key, all);
            last = key;
        }
    }
    if (bad) atomicOr(out.status, CP_STATUS_BAD_TOKEN);
}

// COLUMNS: many tokens a row are summed by place in LDS, each of `lanes` lanes in a column of its own (so that the order of the
// sums is fixed), and the row's columns added up; else every lane looks through all of the row's tokens for its own places.
// `used` (a power of two): of a row's lanes those that take tokens; only these have columns.
template <typename T, typename I, int S, bool COLUMNS>
__global__ __launch_bounds__(kThreads) void few_gradient_kernel(Rows r, Tokens tok, const float *stats, Grads d, T *out, int64_t ldo, int lanes, int used) {
    extern __shared__ float lds_columns[];       // [kWaves][vocab][side * used + 1]
    const int lane = threadIdx.x & (kWave - 1), here = lane & (lanes - 1), group = lane / lanes, side = kWave / lanes;
    const int pitch = side * used + 1, column = group * used + here, log_used = __builtin_ctz(used);
    float *columns = lds_columns + (threadIdx.x / kWave) * (r.vocab * pitch);
    const Few few(r.vocab, lane & (S - 1));
    bool bad = false;
    const int64_t step = (int64_t)gridDim.x * kWaves * side;
    int64_t row0 = ((int64_t)blockIdx.x * kWaves + threadIdx.x / kWave) * side;
    float soon[kEach];
    few.load<T>(soon, r, min(row0 + group, r.rows - 1));
    for (; row0 < r.rows; row0 += step) {
        const int64_t row = min(row0 + group, r.rows - 1);
        const bool live = row0 + group < r.rows;
        float x[kEach], hits[kEach];
#pragma unroll
        for (int e = 0; e < kEach; e++) {
            x[e] = soon[e];
            hits[e] = 0.0f;
        }
        few.load<T>(soon, r, min(row0 + step + group, r.rows - 1));
        if constexpr (COLUMNS) {
            for (int i = here; i < r.vocab * used; i += lanes) columns[(i >> log_used) * pitch + group * used + (i & (used - 1))] = 0.0f;
            lds_ready();
            for (int32_t g0 = here < used ? here * 4 : tok.count; g0 < tok.count; g0 += kAhead * used * 4) {
                Four<I> four[kAhead];
                Pack<float, 4> w[kAhead];
#pragma unroll
                for (int a = 0; a < kAhead; a++) {
                    const int32_t g = g0 + a * used * 4;
                    if (g >= tok.count) continue;
                    four[a].load(tok, row, g);
                    if (d.stride == 1 && g + 4 <= tok.count) w[a] = load_pack<float, 4>(d.dlogp + row * d.row_stride + g);
                    else
#pragma unroll
                        for (int j = 0; j < 4; j++) w[a].v[j] = g + j < tok.count ? d.get(row, g + j) : 0.0f;
                }
#pragma unroll
                for (int a = 0; a < kAhead; a++) {
                    if (g0 + a * used * 4 >= tok.count) continue;
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const int v = four[a].place(j, r.vocab, bad);
                        columns[max(v, 0) * pitch + column] += v >= 0 ? w[a].v[j] : 0.0f;
                    }
                }
            }
            lds_ready();
            // (a place's sum goes where its first column was, which no other lane has read)
            for (int v = here; v < r.vocab; v += lanes) {
                float *from = columns + v * pitch + group * used, sum = 0.0f;
#pragma unroll 8
                for (int j = 0; j < used; j++) sum += from[j];
                from[0] = sum;
            }
            lds_ready();
#pragma unroll
            for (int e = 0; e < kEach; e++) hits[e] = columns[min(few.at + e, r.vocab - 1) * pitch + group * used];
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
        } else {
            for (int32_t g = 0; g < tok.count; g++) {
                const int64_t v = ((const I *)tok.at)[row * tok.row_stride + (int64_t)g * tok.stride];
                const float w = d.get(row, g);
#pragma unroll
                for (int e = 0; e < kEach; e++) hits[e] += v == few.at + e ? w : 0.0f;
            }
        }
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < kEach; e++) {
            hits[e] = x[e] == kNone ? 0.0f : hits[e];
            sum += few.mine >> e & 1 ? hits[e] : 0.0f;
        }
        const Slope slope(r, stats + 3 * row, d.dentropy ? d.dentropy[row * d.de_stride] : 0.0f, group_add<S>(sum));
        if (!live || here >= S || few.mine == 0) continue;
        Pack<T, kEach> o;
#pragma unroll
        for (int e = 0; e < kEach; e++) o.v[e] = (T)slope.at(x[e], hits[e]);
        T *to = out + row * ldo + few.at;
        if (r.vocab >= kEach) store_pack<T, kEach>(to, o);
        else
#pragma unroll
            for (int e = 0; e < kEach; e++)
                if (few.here >> e & 1) to[e] = o.v[e];
    }
}

__global__ void clear_status_kernel(int32_t *status) { *status = CP_STATUS_OK; }

constexpr int kMostLoads = 4;
// Up to so many places a row is some lanes', as many as 32 have room for: 300000 bf16 rows of 200 with one token 101 us forward and
// 96 backward, 350 and 302 in slices of a workgroup each; of 256 111 and 103 (367, 333); 20000 of 256 19 and 11 (29, 23).
constexpr int32_t kFew = CP_LOGPROBS_IN_PLACE;
constexpr size_t kColumnBytes = 72u << 10;   // of LDS for a workgroup's columns: two of them on a compute unit
constexpr int32_t slice_places(int v, int nv) { return kThreads * v * nv; }
int32_t slices_of(int32_t vocab, int v, int nv) { return (vocab + slice_places(v, nv) - 1) / slice_places(v, nv); }

// loads a thread: as many as leave the chip two workgroups a compute unit, and no more than the row has
int loads_of(int64_t rows, int32_t vocab, int v) {
    int nv = 1;
    while (nv < kMostLoads && slice_places(v, nv) < vocab && rows * slices_of(vocab, v, 2 * nv) >= 512) nv *= 2;
    return nv;
}

int check_rows(int64_t rows, int32_t vocab, int type, int32_t given, int token_type) {
    if (!known_type(type) || (given > 0 && token_type != CP_TOKEN_U8 && token_type != CP_TOKEN_I32 && token_type != CP_TOKEN_I64)) return CP_ERR_ARG;
    // (a row's lanes go on by up to kAhead fours each, together 1,024 tokens, and count them in 32 bits)
    static_assert(CP_LOGPROBS_MAX_GIVEN - 1ll + kAhead * 4 * kWave <= INT32_MAX, "the last step ends behind the last token");
    if (rows < 0 || rows > INT32_MAX || vocab < 1 || vocab > CP_LOGPROBS_MAX_VOCAB || given < 0 || given > CP_LOGPROBS_MAX_GIVEN) return CP_ERR_SIZE;
    return CP_OK;
}

// (in units of ln 2 a scale above 2.358e38 is infinite, and a row's largest logit, 0 units from itself, a NaN)
bool scale_fits(float scale) { return scale > 0.0f && scale * kLog2e <= FLT_MAX; }

// workgroups of the finest slicing that a call of these sizes can take
int64_t most_slices(int64_t rows, int32_t vocab) {
    if (vocab <= kFew) return 0;
    return rows * std::max(slices_of(vocab, 4, loads_of(rows, vocab, 4)), slices_of(vocab, 8, loads_of(rows, vocab, 8)));
}

// f(loads a thread)
template <typename F>
int by_loads(int nv, F f) {
    if (nv == 1) return f(std::integral_constant<int, 1>{});
    if (nv == 2) return f(std::integral_constant<int, 2>{});
    return f(std::integral_constant<int, kMostLoads>{});
}

// f(a value of the tokens' type, lanes that have a row's places)
template <typename F>
int by_lanes(const Tokens &tok, int32_t vocab, F f) {
    auto of = [&](auto i) {
        using std::integral_constant;
        if (vocab <= kEach) return f(i, integral_constant<int, 1>{});
        if (vocab <= 2 * kEach) return f(i, integral_constant<int, 2>{});
        if (vocab <= 4 * kEach) return f(i, integral_constant<int, 4>{});
        if (vocab <= 8 * kEach) return f(i, integral_constant<int, 8>{});
        if (vocab <= 16 * kEach) return f(i, integral_constant<int, 16>{});
        return f(i, integral_constant<int, 32>{});
    };
    if (tok.type == CP_TOKEN_U8) return of(uint8_t{});
    if (tok.type == CP_TOKEN_I32) return of(int32_t{});
    return of(int64_t{});
}
static_assert(kFew <= 32 * kEach, "the most lanes have a row's places");

// Lanes of a row with `given` tokens, of which a lane takes four at once: no more than `most`, unless rows do not fill the chip.
int lanes_of(int64_t rows, int32_t given, int least, int most) {
    int lanes = least;
    while (lanes < kWave && lanes * 4 < given && (lanes < most || rows * lanes < (1 << 19))) lanes *= 2;
    return lanes;
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
    if (!scale_fits(scale)) return CP_ERR_ARG;
    if (!status_out) return CP_ERR_NULL;
    if (rows > 0 && (!logits || !entropy || !stats || (given && (!tokens || !logp)) || (top && (!top_logp || !top_idx)))) return CP_ERR_NULL;
    if (rows > 1 && ld < vocab) return CP_ERR_SIZE;
    size_t need = 0;
    cp_token_logprobs_workspace_bytes(rows, vocab, top, &need);
    if (need && !workspace) return CP_ERR_NULL;
    if ((uintptr_t)workspace % kPolicyAlign || workspace_bytes < need) return CP_ERR_WORKSPACE;
    const Extent in = matrix_at(logits, rows, vocab, ld, type);
    if (in_the_way({in}, {vector_at(logp, rows * given), vector_at(entropy, rows), vector_at(stats, 3 * rows), vector_at(top ? top_logp : nullptr, rows * top),
                          vector_at(top ? top_idx : nullptr, rows * top, sizeof(int32_t))}))
        return CP_ERR_ARG;
    const hipStream_t st = (hipStream_t)stream;
    auto clear = [&] { hipLaunchKernelGGL(clear_status_kernel, dim3(1), dim3(1), 0, st, status_out); };
    if (rows == 0) {
        clear();
        return launched();
    }
    const Rows r{rows, vocab, logits, ld, scale, scale * kLog2e, allow, (vocab + 63) / 64};
    const Tokens tok{tokens, token_type, token_row_stride, token_stride, given};
    const Results out{logp, entropy, stats, top_logp, top_idx, top, status_out, (size_t)rows * given * sizeof(float) > kStreamed};
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        if (vocab <= kFew) {
            clear();
            return by_lanes(tok, vocab, [&](auto i, auto l) {
                constexpr int S = decltype(l)::value;
                // (eight lanes write a line of 128 bytes, and many rows share what is done once a row: 646087 rows of 25 with 94
                // tokens take 189 us so, 218 with lanes for all tokens; 200000 rows of 16 with 200 tokens 85 and 103.  Of more
                // tokens the results are written faster line behind line: 200000 rows with 1000 tokens 446 and 186 us, tokens in the caches.)
                const int lanes = lanes_of(rows, given, S, given < 256 ? 8 : kWave), side = kWaves * kWave / lanes;
                hipLaunchKernelGGL((few_kernel<T, decltype(i), S>), dim3((unsigned)std::min<int64_t>((rows + side - 1) / side, 256 * 8)),
                                   dim3(kThreads), 0, st, r, tok, out, lanes);
                return launched();
            });
        }
        constexpr int V = 16 / sizeof(T);
        const int nv = loads_of(rows, vocab, V);
        const int32_t slices = slices_of(vocab, V, nv);
        if (rows * slices > INT32_MAX) return (int)CP_ERR_SIZE;
        Part *parts = (Part *)workspace;
        uint64_t *best = (uint64_t *)((char *)workspace + align_up((size_t)rows * slices * sizeof(Part)));
        if (slices == 1) clear();
        return by_loads(nv, [&](auto n) {
            auto *kernel = top ? slice_kernel<T, V, decltype(n)::value, true> : slice_kernel<T, V, decltype(n)::value, false>;
            hipLaunchKernelGGL(kernel, grid_of(rows * slices), dim3(kThreads), 0, st, r, tok, out, slices, parts, best);
            if (slices > 1) hipLaunchKernelGGL((join_kernel<T>), grid_of(rows), dim3(kThreads), 0, st, r, tok, out, slices, parts, best);
            return launched();
        });
    });
}

int cp_token_logprobs_backward(int64_t rows, int32_t vocab, int type, const void *logits, int64_t ld, float scale, const uint64_t *allow,
                               int32_t given, const void *tokens, int token_type, int64_t token_row_stride, int64_t token_stride,
                               const float *stats, const float *dlogp, int64_t dlogp_row_stride, int64_t dlogp_stride,
                               const float *dentropy, int64_t dentropy_stride, void *dlogits, int64_t ldd, void *stream) {
    int rc = check_rows(rows, vocab, type, given, token_type);
    if (rc) return rc;
    if (!scale_fits(scale)) return CP_ERR_ARG;
    if (rows > 0 && (!logits || !stats || !dlogits || (given && (!tokens || !dlogp)))) return CP_ERR_NULL;
    if (rows > 1 && (ld < vocab || ldd < vocab)) return CP_ERR_SIZE;
    // (a row of few places is read and written by one group of lanes; of many, by workgroups that each read the logits of all its tokens)
    if (in_the_way({matrix_at(logits, rows, vocab, ld, type)}, {matrix_at(dlogits, rows, vocab, ldd, type)}, vocab <= kFew) ||
        in_the_way({vector_at(stats, 3 * rows)}, {matrix_at(dlogits, rows, vocab, ldd, type)}))
        return CP_ERR_ARG;
    if (rows == 0) return CP_OK;
    const Rows r{rows, vocab, logits, ld, scale, scale * kLog2e, allow, (vocab + 63) / 64};
    const Tokens tok{tokens, token_type, token_row_stride, token_stride, given};
    const Grads d{dlogp, dlogp_row_stride, dlogp_stride, dentropy, dentropy_stride};
    const hipStream_t st = (hipStream_t)stream;
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        if (vocab <= kFew)
            return by_lanes(tok, vocab, [&](auto i, auto l) {
                constexpr int S = decltype(l)::value;
                using I = decltype(i);
                // (Columns have to be cleared and added up; without them each of S lanes reads all tokens.  us in columns and without,
                // 300000 rows: of 8 places with 16 tokens of a byte 20 and 12, with 32 31 and 26, with 64 33 and 45; with 16 of eight
                // bytes 21 and 30, with 32 34 and 66.  Of 25 places with 24 tokens of a byte 45 and 39, with 48 48 and 59; of 64 with 48
                // 125 and 117, with 96 135 and 193.)
                const bool sums = given >= (S <= 2 ? 16 : 48);
                const int lanes = sums ? lanes_of(rows, given, S, 8) : S, side = kWaves * kWave / lanes;
                const dim3 grid((unsigned)std::min<int64_t>((rows + side - 1) / side, 256 * 8));
                int used = 1;
                while (used < lanes && used * 4 < given) used *= 2;
                auto bytes = [&] { return sums ? (size_t)kWaves * vocab * (kWave / lanes * used + 1) * sizeof(float) : 0; };
                while (used > 1 && bytes() > kColumnBytes) used /= 2;
                const size_t lds = bytes();
                auto *kernel = sums ? few_gradient_kernel<T, I, S, true> : few_gradient_kernel<T, I, S, false>;
                if (lds > 48 * 1024 && hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
                    return (int)CP_ERR_HIP;
                hipLaunchKernelGGL(kernel, grid, dim3(kThreads), lds, st, r, tok, stats, d, (T *)dlogits, ldd, lanes, used);
                return launched();
            });
        constexpr int V = 16 / sizeof(T);
        const int nv = loads_of(rows, vocab, V);
        const int32_t slices = slices_of(vocab, V, nv);
        if (rows * slices > INT32_MAX) return (int)CP_ERR_SIZE;
        return by_loads(nv, [&](auto n) {
            hipLaunchKernelGGL((gradient_kernel<T, V, decltype(n)::value>), grid_of(rows * slices), dim3(kThreads), 0, st, r, tok, stats, d,
                               (T *)dlogits, ldd, slices, (size_t)rows * vocab * sizeof(T) > kStreamed);
            return launched();
        });
    });
}

}  // extern "C"
