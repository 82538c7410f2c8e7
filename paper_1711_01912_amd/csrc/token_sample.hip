// Tokens drawn from rows of logits by given random numbers, with temperature, top-k, top-p and min-p:
//
//   p_v = exp((x_v - max x) scale) over the allowed places, in the order of falling x (ties: the lower place)
//   kept: the first top_k places; of these those in front of which less than top_p of their mass lies; of these p_v >= min_p
//   token = the first kept place, by place, up to and with which more than u of the kept mass lies
//
// The kept places are a beginning of that order: all above a logit, and the first few of those that equal it.  What is drawn is
// a place, not a value that may be off by a rounding: probabilities and their sums are formed in 64 bits (on this chip
// at the rate of 32), so that a draw differs from the definition only where u lies within 1e-12 of a border.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <climits>

#include "policy.hpp"

namespace cpeval {

namespace {

struct Settings {
    double scale, top_p, min_p;
    int32_t top_k;                       // 0: all
    const float *scales, *top_ps, *min_ps;
    const int32_t *top_ks;               // [rows] each, or null
};

struct Draw {
    int64_t rows;
    int32_t vocab, words;                // words of a row's mask
    const void *logits;
    int64_t ld;
    const uint64_t *allow;
    Settings set;
    int32_t given;
    const float *u;
    int64_t u_row, u_step;
    void *tokens;
    int token_type;
    int64_t t_row, t_step;
    float *logp;                         // [rows][given], or null
    int32_t *status;
};

// one row's settings; false: out of range
struct Rule {
    double scale, top_p, min_p;
    int32_t top_k;
    bool fine;
    __device__ __forceinline__ bool sorts() const { return top_k > 0 || top_p < 1.0; }
};
__device__ __forceinline__ Rule rule_of(const Settings &s, int64_t row) {
    Rule r;
    r.scale = s.scales ? (double)s.scales[row] : s.scale;
    r.top_p = s.top_ps ? (double)s.top_ps[row] : s.top_p;
    r.min_p = s.min_ps ? (double)s.min_ps[row] : s.min_p;
    r.top_k = s.top_ks ? s.top_ks[row] : s.top_k;
    r.fine = r.scale > 0.0 && r.scale <= FLT_MAX && r.top_p >= 0.0 && r.top_p <= 1.0 && r.min_p >= 0.0 && r.min_p <= 1.0 && r.top_k >= 0;
    return r;
}

__device__ __forceinline__ void put_token(const Draw &d, int64_t row, int32_t g, int32_t token) {
    const int64_t at = row * d.t_row + g * d.t_step;
    if (d.token_type == 1) ((uint8_t *)d.tokens)[at] = (uint8_t)token;
    else if (d.token_type == 4) ((int32_t *)d.tokens)[at] = token;
    else ((int64_t *)d.tokens)[at] = token;
}

// Row's g-th random number.  Below 0, and NaN, it counts as 0, from 1 on as the last number below 1.
__device__ __forceinline__ float number(const Draw &d, int64_t row, int32_t g) {
    return fminf(fmaxf(d.u[row * d.u_row + g * d.u_step], 0.0f), 0x1.fffffep-1f);
}

// the first float that is not below v >= 0
__device__ __forceinline__ float float_above(double v) {
    const float f = (float)v;
    return (double)f < v ? __uint_as_float(__float_as_uint(f) + 1) : f;
}

// larger logits have larger keys, equal ones (0 and -0) the same
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

template <int L>
__device__ __forceinline__ float most_of(float v) {
#pragma unroll
    for (int off = L / 2; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}
template <int L>
__device__ __forceinline__ double sum_of(double v) {
#pragma unroll
    for (int off = L / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}
// the sum of the lanes up to and with one's own, in groups of L
template <int L>
__device__ __forceinline__ double sum_upto(double v, int lane) {
#pragma unroll
    for (int off = 1; off < L; off <<= 1) {
        const double o = __shfl_up(v, off);
        if (lane % L >= off) v += o;
    }
    return v;
}

// ---- rows of few places ------------------------------------------------------------------------------

constexpr int kFew = 256, kFewThreads = 256;

// L lanes a row, places 4 lane .. 4 lane + 3 of each where there are more than L, else one each.  A row's borders, cumulated
// shares of its mass, are rounded up to floats: u, a float, is below one just if it is below the other.  A draw then is the number of borders
// that are not above u.
template <typename T, int L>
__global__ __launch_bounds__(kFewThreads) void few_sample_kernel(Draw d) {
    constexpr int kRowsHere = kFewThreads / L, kPer = L == 64 ? 4 : 1, kRoom = L * kPer;
    __shared__ float border[kRowsHere][kRoom + 1], lp[kRowsHere][kRoom + 1], xs[kRowsHere][kRoom + 1];
    __shared__ double ps[kRowsHere][kRoom];
    const int lane = threadIdx.x % L, mine = threadIdx.x / L;
    const int64_t row = (int64_t)group_number() * kRowsHere + mine;
    const bool here = row < d.rows;
    const int V = d.vocab;
    const int per = kPer == 1 ? 1 : (V + L - 1) / L;
    Rule rule{1.0, 1.0, 0.0, 0, false};
    float x[kPer];
    float m = -INFINITY;
    bool odd = false;
    if (here) rule = rule_of(d.set, row);
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        const int v = lane * per + i;
        x[i] = -INFINITY;
        if (here && i < per && v < V) {
            const float at = (float)((const T *)d.logits)[row * d.ld + v];
            const bool open = !d.allow || (d.allow[row * d.words + (v >> 6)] >> (v & 63) & 1);
            if (open) {
                x[i] = at;
                odd |= !(at < INFINITY);
            }
        }
        m = fmaxf(m, x[i]);
    }
    m = most_of<L>(m);
    const uint64_t odds = __ballot(odd);
    const uint64_t group = L == 64 ? ~0ull : ((1ull << (L & 63)) - 1) << (threadIdx.x % kWave / L * L);
    const bool none = !here || m == -INFINITY || (odds & group) || !rule.fine;
    if (here && !rule.fine && lane == 0) atomicOr(d.status, CP_STATUS_BAD_SAMPLING);
    double p[kPer];
#pragma unroll
    for (int i = 0; i < kPer; i++) p[i] = none || x[i] == -INFINITY ? 0.0 : exp(((double)x[i] - (double)m) * rule.scale);
    const bool sorts = !none && rule.sorts();
    if (sorts) {
#pragma unroll
        for (int i = 0; i < kPer; i++) {
            const int v = lane * per + i;
            if (i < per && v < V) xs[mine][v] = x[i], ps[mine][v] = p[i];
        }
    }
    __syncthreads();
    if (sorts) {
        // how many places, and how much of the mass, lie in front of each
        int rank[kPer];
        double ahead[kPer], total = 0;
#pragma unroll
        for (int i = 0; i < kPer; i++) rank[i] = 0, ahead[i] = 0;
        for (int j = 0; j < V; j++) {
            const float xj = xs[mine][j];
            const double pj = ps[mine][j];
#pragma unroll
            for (int i = 0; i < kPer; i++) {
                const int v = lane * per + i;
                const bool front = xj > x[i] || (xj == x[i] && j < v);
                rank[i] += front;
                ahead[i] += front ? pj : 0.0;
            }
        }
#pragma unroll
        for (int i = 0; i < kPer; i++) {
            if (rule.top_k > 0 && rank[i] >= rule.top_k) p[i] = 0;
            total += p[i];
        }
        total = sum_of<L>(total) * rule.top_p;
#pragma unroll
        for (int i = 0; i < kPer; i++)
            if (rule.top_p < 1.0 && rank[i] > 0 && !(ahead[i] < total)) p[i] = 0;
    }
    double upto = 0;
    int last = -1;
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        if (p[i] < rule.min_p) p[i] = 0;
        upto += p[i];
        if (p[i] > 0) last = lane * per + i;
    }
    const double total = sum_of<L>(upto);
    double sum = sum_upto<L>(upto, lane) - upto;
#pragma unroll
    for (int off = L / 2; off > 0; off >>= 1) last = max(last, __shfl_xor(last, off));
    const double logs = d.logp && !none ? log(total) : 0.0;
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        const int v = lane * per + i;
        sum += p[i];
        if (i < per && v < V) {
            // (the last place that can be drawn takes what rounding leaves)
            border[mine][v] = v >= last ? INFINITY : float_above(sum / total);
            if (d.logp) lp[mine][v] = (float)(((double)x[i] - (double)m) * rule.scale - logs);
        }
    }
    __syncthreads();
    if (!here) return;
    const float *edge = border[mine];
    float at[15];
#pragma unroll
    for (int v = 0; v < 15; v++) at[v] = v < V - 1 ? edge[v] : INFINITY;
    auto draw = [&](float u) {
        int n = 0, hi = V - 1;               // the first border above u
        if (V <= 16) {
#pragma unroll
            for (int v = 0; v < 15; v++) n += !(u < at[v]);
            return n;
        }
        while (n < hi) {
            const int mid = (n + hi) / 2;
            if (!(u < edge[mid])) n = mid + 1;
            else hi = mid;
        }
        return n;
    };
    for (int32_t g = lane; g < d.given; g += L) {
        int token = -1;
        if (!none) token = draw(number(d, row, g));
        put_token(d, row, g, token);
        if (d.logp) d.logp[row * d.given + g] = none ? 0.0f : lp[mine][token];
    }
}

// ---- rows of many places -----------------------------------------------------------------------------

constexpr int kManyThreads = 1024, kManyWaves = kManyThreads / kWave;
constexpr int kBins = 2048, kChunks = 2048;

// sums over the threads in front of one's own; total of all
template <typename N>
__device__ __forceinline__ N block_before(N v, N *room, N &total) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    N upto = v;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const N o = __shfl_up(upto, off);
        if (lane >= off) upto += o;
    }
    __syncthreads();
    if (lane == kWave - 1) room[wave] = upto;
    __syncthreads();
    N before = 0;
    total = 0;
    for (int w = 0; w < kManyWaves; w++) {
        if (w < wave) before += room[w];
        total += room[w];
    }
    return before + upto - v;
}

// A workgroup a row, which is read from the caches for each of: the maximum; the logit that top_k and top_p end at, digit by digit of its
// key from a histogram of places or of mass (in whole numbers, which add up the same in any order); the mass of each chunk; the draws.
template <typename T>
struct Many {
    static constexpr int kVec = 16 / (int)sizeof(T), kStep = kWave * kVec;      // places of a lane and of a wavefront's load
    static constexpr int kLevels = sizeof(T) == 2 ? 2 : 3, kDrop = sizeof(T) == 2 ? 10 : 0;        // digits of 11, 11 and 10 bits

    const T *row;
    const uint64_t *allow;
    int32_t V;
    float m;
    double scale;

    // kVec places from v on; what is not there or not allowed is -inf
    __device__ __forceinline__ void load(int32_t v, float (&x)[kVec]) const {
        uint64_t bits = ~0ull;
        if (allow && v < V) bits = allow[v >> 6] >> (v & 63);
        if (v + kVec <= V) {
            const Pack<T, kVec> at = load_pack<T, kVec>(row + v);
#pragma unroll
            for (int i = 0; i < kVec; i++) x[i] = bits >> i & 1 ? (float)at.v[i] : -INFINITY;
        } else {
#pragma unroll
            for (int i = 0; i < kVec; i++) x[i] = v + i < V && (bits >> i & 1) ? (float)row[v + i] : -INFINITY;
        }
    }
    __device__ __forceinline__ double share(float x) const { return x == -INFINITY ? 0.0 : exp(((double)x - (double)m) * scale); }
    __device__ __forceinline__ static uint32_t key(float x) { return order_key(x) >> kDrop; }
    __device__ __forceinline__ static float value(uint32_t key) {
        uint32_t b = key << kDrop;
        if (b & 0x80000000u) b &= 0x7fffffffu;
        else b = ~(b | ((1u << kDrop) - 1));
        return __uint_as_float(b);
    }
    __device__ __forceinline__ static int shift(int level) { return kLevels == 2 ? 11 - 11 * level : 21 - 11 * level + (level == 2); }
};

template <typename T>
__global__ __launch_bounds__(kManyThreads) void many_sample_kernel(Draw d) {
    using M = Many<T>;
    constexpr int kVec = M::kVec, kStep = M::kStep;
    __shared__ uint64_t bins[kBins];
    __shared__ double mass[kChunks];
    __shared__ int32_t ties[kChunks];
    __shared__ union { float f[kManyWaves]; uint64_t u[kManyWaves]; double d[kManyWaves]; int32_t i[kManyWaves]; } room;
    __shared__ int odd_, found_bin;
    __shared__ uint64_t found_above;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t row = group_number();
    if (row >= d.rows) return;
    Rule rule = rule_of(d.set, row);
    if (rule.top_p == 0.0) rule.top_p = 1.0, rule.top_k = 1;       // (the best alone)
    M a{(const T *)d.logits + row * d.ld, d.allow ? d.allow + row * d.words : nullptr, d.vocab, 0.0f, rule.scale};
    const int32_t V = d.vocab;

    if (threadIdx.x == 0) odd_ = 0;
    __syncthreads();
    float m = -INFINITY;
    bool odd = false;
    for (int64_t v = (int64_t)threadIdx.x * kVec; v < V; v += kManyThreads * kVec) {
        float x[kVec];
        a.load((int32_t)v, x);
#pragma unroll
        for (int i = 0; i < kVec; i++) odd |= !(x[i] < INFINITY), m = fmaxf(m, x[i]);
    }
    m = most_of<kWave>(m);
    if (lane == 0) room.f[wave] = m;
    if (odd) odd_ = 1;
    __syncthreads();
    for (int w = 0; w < kManyWaves; w++) m = fmaxf(m, room.f[w]);
    a.m = m;
    if (odd_ || m == -INFINITY || !rule.fine) {
        if (!rule.fine && threadIdx.x == 0) atomicOr(d.status, CP_STATUS_BAD_SAMPLING);
        for (int32_t g = threadIdx.x; g < d.given; g += kManyThreads) {
            put_token(d, row, g, -1);
            if (d.logp) d.logp[row * d.given + g] = 0.0f;
        }
        return;
    }

    // The place in the order where what is kept ends: keys above `key_end`, and `keep_ties` of those that equal it
    uint32_t key_end = 0;
    int64_t keep_ties = INT64_MAX;
    // finds the bin, from the highest on, in which the weight reaches `want` (past what lies above the bins)
    auto seek = [&](double want, uint64_t above) {
        // (thread t has the t-th pair of bins from the top)
        const int top = kBins - 1 - 2 * (int)threadIdx.x;
        const uint64_t first = bins[top], second = bins[top - 1];
        uint64_t total;
        const uint64_t before = above + block_before<uint64_t>(first + second, room.u, total);
        if (threadIdx.x == 0) found_bin = 0, found_above = above + total;      // (rounding: the lowest)
        __syncthreads();
        if ((double)before < want && !((double)(before + first + second) < want)) {
            const bool one = !((double)(before + first) < want);
            found_bin = one ? top : top - 1, found_above = one ? before : before + first;
        }
        __syncthreads();
        return total;
    };
    auto clear = [&] {
        __syncthreads();
        for (int i = threadIdx.x; i < kBins; i += kManyThreads) bins[i] = 0;
        __syncthreads();
    };
    if (rule.top_k > 0 && rule.top_k < V) {
        uint64_t above = 0;
        uint32_t prefix = 0;
        for (int level = 0; level < M::kLevels; level++) {
            const int sh = M::shift(level), width = level == 2 ? 10 : 11;
            clear();
            for (int64_t v = (int64_t)threadIdx.x * kVec; v < V; v += kManyThreads * kVec) {
                float x[kVec];
                a.load((int32_t)v, x);
#pragma unroll
                for (int i = 0; i < kVec; i++) {
                    const uint32_t k = M::key(x[i]);
                    if (v + i < V && (level == 0 || k >> (sh + width) == prefix)) atomicAdd((unsigned int *)&bins[k >> sh & ((1u << width) - 1)], 1u);
                }
            }
            __syncthreads();
            seek((double)rule.top_k, above);
            prefix = prefix << width | (uint32_t)found_bin, above = found_above;
            __syncthreads();
        }
        key_end = prefix, keep_ties = (int64_t)rule.top_k - (int64_t)above;
    }
    if (rule.top_p < 1.0) {
        // mass in units so small that a sum of all places stays below 2^62
        const double unit = ldexp(1.0, 62 - (32 - __clz(V)));
        const uint32_t least = key_end;
        const int64_t least_ties = keep_ties;
        uint64_t above = 0;
        uint32_t prefix = 0;
        double want = 0;
        for (int level = 0; level < M::kLevels; level++) {
            const int sh = M::shift(level), width = level == 2 ? 10 : 11;
            clear();
            for (int64_t v = (int64_t)threadIdx.x * kVec; v < V; v += kManyThreads * kVec) {
                float x[kVec];
                a.load((int32_t)v, x);
#pragma unroll
                for (int i = 0; i < kVec; i++) {
                    const uint32_t k = M::key(x[i]);
                    // (of those that equal the last of the top_k, added below, only some are left)
                    if (x[i] > -INFINITY && (k > least || least_ties == INT64_MAX) && (level == 0 || k >> (sh + width) == prefix))
                        atomicAdd((unsigned long long *)&bins[k >> sh & ((1u << width) - 1)], (unsigned long long)(a.share(x[i]) * unit + 0.5));
                }
            }
            __syncthreads();
            if (threadIdx.x == 0 && least_ties != INT64_MAX && (level == 0 || least >> (sh + width) == prefix))
                bins[least >> sh & ((1u << width) - 1)] += (uint64_t)least_ties * (uint64_t)(a.share(M::value(least)) * unit + 0.5);
            __syncthreads();
            if (level == 0) {
                uint64_t total = 0;
                block_before<uint64_t>(bins[2 * threadIdx.x] + bins[2 * threadIdx.x + 1], room.u, total);
                want = (double)total * rule.top_p;
            }
            seek(want, above);
            prefix = prefix << width | (uint32_t)found_bin, above = found_above;
            __syncthreads();
        }
        // places that equal the last one: as long as less than `want` lies in front of them, the first in any case
        const uint64_t each = (uint64_t)(a.share(M::value(prefix)) * unit + 0.5);
        int64_t more = V;
        if (each > 0) {
            more = max((int64_t)(((double)want - (double)above) / (double)each), (int64_t)0);
            while (more > 0 && !((double)(above + (uint64_t)(more - 1) * each) < want)) more--;
            while ((double)(above + (uint64_t)more * each) < want) more++;
        }
        more = max(more, (int64_t)(above == 0));
        if (prefix == least) more = min(more, least_ties);
        key_end = prefix, keep_ties = more;
    }
    // what equals the last one and is less likely than min_p goes too
    const double end_share = keep_ties == INT64_MAX ? 0.0 : a.share(M::value(key_end));
    if (keep_ties != INT64_MAX && end_share < rule.min_p) keep_ties = 0;
    const bool cut = keep_ties != INT64_MAX;

    // The row in chunks, one after the other, a wavefront each: mass above the end, and how many equal it
    const int32_t steps = (int32_t)(((int64_t)V + (int64_t)kStep * kChunks - 1) / ((int64_t)kStep * kChunks));       // of a chunk
    const int64_t size = (int64_t)steps * kStep;
    const int32_t chunks = (int32_t)((V + size - 1) / size);
    auto kept = [&](float x, bool &tie) {
        tie = false;
        if (x == -INFINITY) return 0.0;
        if (cut) {
            const uint32_t k = M::key(x);
            tie = k == key_end;
            if (k <= key_end) return 0.0;
        }
        const double p = a.share(x);
        return p < rule.min_p ? 0.0 : p;
    };
    for (int32_t c = wave; c < chunks; c += kManyWaves) {
        double sum = 0;
        int32_t same = 0;
        for (int32_t s = 0; s < steps; s++) {
            const int64_t v = c * size + s * kStep + lane * kVec;
            if (v >= V) break;
            float x[kVec];
            a.load((int32_t)v, x);
#pragma unroll
            for (int i = 0; i < kVec; i++) {
                bool tie;
                sum += kept(x[i], tie);
                same += tie;
            }
        }
        sum = sum_of<kWave>(sum);
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) same += __shfl_xor(same, off);
        if (lane == 0) mass[c] = sum, ties[c] = same;
    }
    __syncthreads();
    // of the ties, the first ones by place
    const int32_t c0 = 2 * threadIdx.x, c1 = c0 + 1;
    int32_t t0 = c0 < chunks ? ties[c0] : 0, t1 = c1 < chunks ? ties[c1] : 0, all_ties;
    const int32_t ties_before = block_before<int32_t>(t0 + t1, room.i, all_ties);
    double m0 = c0 < chunks ? mass[c0] : 0, m1 = c1 < chunks ? mass[c1] : 0;
    if (cut) {
        m0 += (double)max(min((int64_t)t0, keep_ties - ties_before), (int64_t)0) * end_share;
        m1 += (double)max(min((int64_t)t1, keep_ties - ties_before - t0), (int64_t)0) * end_share;
    }
    double total;
    const double mass_before = block_before<double>(m0 + m1, room.d, total);
    if (c0 < chunks) mass[c0] = mass_before + m0, ties[c0] = ties_before;
    if (c1 < chunks) mass[c1] = mass_before + m0 + m1, ties[c1] = ties_before + t0;
    __syncthreads();
    const double logs = d.logp ? log(total) : 0.0;

    for (int32_t g = wave; g < d.given; g += kManyWaves) {
        const double target = (double)number(d, row, g) * total;
        int32_t lo = 0, hi = chunks - 1;     // the first chunk that reaches beyond, or the last
        while (lo < hi) {
            const int32_t mid = (lo + hi) / 2;
            if (mass[mid] > target) hi = mid;
            else lo = mid + 1;
        }
        int32_t token = -1, last = -1;
        // (one chunk, unless sums in another order put a border on its other side)
        for (; lo < chunks && token < 0; lo++) {
            double before = lo > 0 ? mass[lo - 1] : 0.0;
            int64_t tie = ties[lo];
            for (int32_t s = 0; s < steps && token < 0; s++) {
                const int64_t v = lo * size + s * kStep + lane * kVec;
                float x[kVec];
                double p[kVec], sum = 0;
                int32_t same = 0;
                bool t[kVec];
                a.load((int32_t)min(v, (int64_t)V), x);
#pragma unroll
                for (int i = 0; i < kVec; i++) {
                    p[i] = kept(x[i], t[i]);
                    same += t[i];
                }
                if (cut) {
                    int32_t upto = same;
#pragma unroll
                    for (int off = 1; off < kWave; off <<= 1) {
                        const int32_t o = __shfl_up(upto, off);
                        if (lane >= off) upto += o;
                    }
                    int64_t rank = tie + upto - same;
#pragma unroll
                    for (int i = 0; i < kVec; i++)
                        if (t[i]) p[i] = rank++ < keep_ties ? end_share : 0.0;
                    tie += __shfl(upto, kWave - 1);
                }
                int32_t hit = -1;
#pragma unroll
                for (int i = 0; i < kVec; i++) {
                    sum += p[i];
                    if (p[i] > 0) hit = (int32_t)v + i;
                }
                last = max(last, hit);
                const double upto = sum_upto<kWave>(sum, lane);
                const uint64_t beyond = __ballot(before + upto > target && sum > 0);
                if (beyond) {
                    double at = before + (upto - sum);
#pragma unroll
                    for (int i = kVec - 1; i >= 0; i--) {
                        // (from the back: the first place that reaches beyond is the last one seen)
                        double here = at;
#pragma unroll
                        for (int k = 0; k <= i; k++) here += p[k];
                        if (p[i] > 0 && here > target) hit = (int32_t)v + i;
                    }
                    token = __shfl(hit, __ffsll((unsigned long long)beyond) - 1);
                }
                before += __shfl(upto, kWave - 1);
            }
        }
        if (token < 0) {
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) last = max(last, __shfl_xor(last, off));
            token = last;
        }
        if (lane == 0) {
            put_token(d, row, g, token);
            if (d.logp) {
                const float x = (float)((const T *)d.logits)[row * d.ld + max(token, 0)];
                d.logp[row * d.given + g] = (float)(((double)x - (double)m) * rule.scale - logs);
            }
        }
    }
}

constexpr int64_t kFar = 1ll << 28;          // strides; products of these, rows and bytes stay in 64 bits

__global__ void clear_sampling_kernel(int32_t *status) { *status = CP_STATUS_OK; }

}  // namespace

}  // namespace cpeval

using namespace cpeval;

extern "C" {

int cp_token_sample_workspace_bytes(int64_t rows, int32_t vocab, int32_t given, size_t *out_bytes) {
    if (!out_bytes) return CP_ERR_NULL;
    if (rows < 0 || rows > INT32_MAX || vocab < 1 || vocab > CP_LOGPROBS_MAX_VOCAB || given < 0 || given > CP_LOGPROBS_MAX_GIVEN) return CP_ERR_SIZE;
    *out_bytes = 0;
    return CP_OK;
}

int cp_token_sample(int64_t rows, int32_t vocab, int type, const void *logits, int64_t ld, double scale, const float *scales,
                    const uint64_t *allow, int32_t top_k, const int32_t *top_ks, double top_p, const float *top_ps, double min_p,
                    const float *min_ps, int32_t given, const float *u, int64_t u_row_stride, int64_t u_stride, void *tokens, int token_type,
                    int64_t token_row_stride, int64_t token_stride, float *logp, void *workspace, size_t workspace_bytes, void *stream,
                    int32_t *status_out) {
    if (!known_type(type) || (token_type != CP_TOKEN_U8 && token_type != CP_TOKEN_I32 && token_type != CP_TOKEN_I64)) return CP_ERR_ARG;
    if ((!scales && !(scale > 0.0 && scale <= FLT_MAX)) || (!top_ks && top_k < 0) || (!top_ps && !(top_p >= 0.0 && top_p <= 1.0)) ||
        (!min_ps && !(min_p >= 0.0 && min_p <= 1.0)))
        return CP_ERR_ARG;
    size_t need = 0;
    const int rc = cp_token_sample_workspace_bytes(rows, vocab, given, &need);
    if (rc) return rc;
    if ((token_type == CP_TOKEN_U8 && vocab > 255) || (rows > 1 && ld < vocab)) return CP_ERR_SIZE;
    const bool own = scales || top_ks || top_ps || min_ps;
    if ((rows > 0 && !logits) || (rows > 0 && given > 0 && (!u || !tokens)) || (own && !status_out)) return CP_ERR_NULL;
    if (rows > 0 && given > 0) {
        // numbers may lie anywhere, tokens apart from each other
        if (u_row_stride < 0 || u_stride < 0 || u_row_stride > kFar || u_stride > kFar || token_row_stride > kFar || token_stride > kFar) return CP_ERR_SIZE;
        const bool apart = token_row_stride >= (given - 1) * token_stride + 1, between = token_stride >= (rows - 1) * token_row_stride + 1;
        if ((given > 1 && token_stride < 1) || (rows > 1 && token_row_stride < 1) || (given > 1 && rows > 1 && !apart && !between)) return CP_ERR_SIZE;
        const int64_t each = token_type, t_row = rows > 1 ? token_row_stride : 0, t_step = given > 1 ? token_stride : 0;
        const Extent to = rows == 1   ? Extent{tokens, 1, ((given - 1) * t_step + 1) * each, 0, (size_t)each}
                          : given == 1 || apart ? Extent{tokens, rows, ((given - 1) * t_step + 1) * each, t_row * each, (size_t)each}
                                                : Extent{tokens, given, ((rows - 1) * t_row + 1) * each, t_step * each, (size_t)each};
        const Extent numbers = vector_at(u, (rows - 1) * u_row_stride + (given - 1) * u_stride + 1);
        if (in_the_way({matrix_at(logits, rows, vocab, ld, type), numbers, vector_at(allow, rows * ((vocab + 63) / 64), 8), vector_at(scales, rows),
                        vector_at(top_ks, rows), vector_at(top_ps, rows), vector_at(min_ps, rows)},
                       {to, vector_at(logp, rows * given), vector_at(own ? status_out : nullptr, 1)}))
            return CP_ERR_ARG;
    }
    const hipStream_t st = (hipStream_t)stream;
    if (own) hipLaunchKernelGGL(clear_sampling_kernel, dim3(1), dim3(1), 0, st, status_out);
    if (rows == 0 || given == 0) return launched();
    const Draw d{rows, vocab, (vocab + 63) / 64, logits, ld, allow, {scale, top_p, min_p, top_k, scales, top_ps, min_ps, top_ks}, given, u,
                 u_row_stride, u_stride, tokens, token_type, token_row_stride, token_stride, logp, status_out};
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        if (vocab > kFew) {
            hipLaunchKernelGGL(many_sample_kernel<T>, grid_of(rows), dim3(kManyThreads), 0, st, d);
            return launched();
        }
        auto go = [&](auto l) {
            constexpr int L = decltype(l)::value;
            hipLaunchKernelGGL((few_sample_kernel<T, L>), grid_of((rows + kFewThreads / L - 1) / (kFewThreads / L)), dim3(kFewThreads), 0, st, d);
            return launched();
        };
        if (vocab <= 8 && given <= 32) return go(std::integral_constant<int, 8>{});
        if (vocab <= 16 && given <= 64) return go(std::integral_constant<int, 16>{});
        if (vocab <= 32 && given <= 128) return go(std::integral_constant<int, 32>{});
        return go(std::integral_constant<int, 64>{});
    });
}

}  // extern "C"
