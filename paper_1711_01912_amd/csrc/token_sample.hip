// Tokens drawn from rows of logits by given random numbers, with temperature, top-k, top-p and min-p:
//
//   p_v = exp((x_v - max x) scale) over the allowed places, in the order of falling x (ties: the lower place)
//   kept: the first top_k places; of these those in front of which less than top_p of their mass lies; of these p_v >= min_p
//   token = the first kept place, by place, up to and with which more than u of the kept mass lies
//
// The kept places are a beginning of that order: all above a logit, and the first few of those that equal it.  What is drawn is
// a place, not a value that may be off by a rounding: probabilities and their sums are formed in 64 bits (on this chip
// at the rate of 32), so that a draw differs from the definition only where u or top_p lies within 1e-12 of a border (top_p 2e-12 in
// rows of 2^26 places).
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
    // of rows that are cut into slices, or 0: what each found
    int32_t slices, slice_size;
    uint64_t *found;                     // [rows][slices][kSliced] words of a list, the largest first
    int32_t *counts;                     // [rows][slices]: how many; or that they had no room, or that there is a NaN or +inf
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

// A random number below 0, and NaN, counts as 0, from 1 on as the last number below 1.
__device__ __forceinline__ float counted(float u) { return fminf(fmaxf(u, 0.0f), 0x1.fffffep-1f); }

// the first float that is not below v >= 0
__device__ __forceinline__ float float_above(double v) {
    const float f = (float)v;
    return (double)f < v ? __uint_as_float(__float_as_uint(f) + 1) : f;
}

// 2^(t + up) for t <= 0 with the relative error of a few roundings of 64 bits: Taylor's polynomial of 2^f, |f| <= 1/2, is off by 0.35^12 / 12! = 7e-15
__device__ __forceinline__ double power_of_two(double t, int up = 0) {
    const double n = __builtin_rint(fmax(t, -1080.0)), f = (fmax(t, -1080.0) - n) * 0.69314718055994530942;
    double p = 1.0 / 39916800;
    p = fma(p, f, 1.0 / 3628800);
    p = fma(p, f, 1.0 / 362880);
    p = fma(p, f, 1.0 / 40320);
    p = fma(p, f, 1.0 / 5040);
    p = fma(p, f, 1.0 / 720);
    p = fma(p, f, 1.0 / 120);
    p = fma(p, f, 1.0 / 24);
    p = fma(p, f, 1.0 / 6);
    p = fma(p, f, 0.5);
    p = fma(p, f, 1.0);
    p = fma(p, f, 1.0);
    return ldexp(p, (int)n + up);
}
constexpr double kLog2eWide = 1.44269504088896340736;

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

// The row's draws, `side` of them side by side from `first` on.  Their number of borders that are not above u: counted where there are few, else by
// halving.
template <typename TT, int E>
__device__ __forceinline__ void draw_more(const Draw &d, int64_t row, const float *edge, const float *lp, bool none, int32_t first, int32_t side) {
    const int V = d.vocab;
    const bool neighbours = d.u_step == 1 && d.t_step == 1;
    float at[E > 0 ? E : 1];
#pragma unroll
    for (int v = 0; v < E; v++) at[v] = v < V - 1 ? edge[v] : INFINITY;
    const auto draw = [&](float u) {
        int n = 0;
        if constexpr (E > 0) {
#pragma unroll
            for (int v = 0; v < E; v++) n += !(u < at[v]);
        } else {
            int hi = V - 1;                  // the first border above u
            while (n < hi) {
                const int mid = (n + hi) / 2;
                if (!(u < edge[mid])) n = mid + 1;
                else hi = mid;
            }
        }
        return n;
    };
    TT *to = (TT *)d.tokens + row * d.t_row;
    const float *u = d.u + row * d.u_row;
    float *logp = d.logp ? d.logp + row * d.given : nullptr;
    int32_t done = 0;
    if (neighbours && side == kWave) {
        // four neighbouring draws a lane
        for (int32_t g = 4 * first; g + 4 <= d.given; g += 4 * side) {
            const Pack<float, 4> four = load_pack<float, 4>(u + g);
            Pack<TT, 4> token;
            Pack<float, 4> l;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int n = none ? -1 : draw(counted(four.v[e]));
                token.v[e] = (TT)n;
                if (logp) l.v[e] = none ? 0.0f : lp[n];
            }
            store_pack<TT, 4>(to + g, token);
            if (logp) store_pack<float, 4>(logp + g, l);
        }
        done = d.given & ~3;
    }
    for (int32_t g = done + first; g < d.given; g += side) {
        const int n = none ? -1 : draw(counted(u[g * d.u_step]));
        to[g * d.t_step] = (TT)n;
        if (logp) logp[g] = none ? 0.0f : lp[n];
    }
}
template <typename TT>
__device__ __forceinline__ void draw_row(const Draw &d, int64_t row, const float *edge, const float *lp, bool none, int32_t first, int32_t side) {
    if (d.vocab <= 8) draw_more<TT, 7>(d, row, edge, lp, none, first, side);
    else if (d.vocab <= 16) draw_more<TT, 15>(d, row, edge, lp, none, first, side);
    else draw_more<TT, 0>(d, row, edge, lp, none, first, side);
}

// L lanes a row, PER neighbouring places each at most.  Places are put in order by counting those in front of each, which bounds rows that are
// cut and have few draws (5,271 rows of 50 with 333 draws 23 us; 38 with 16 lanes of four places a row).  A row's borders, cumulated shares
// of its mass, are rounded up to floats: u, a float, is below one just if it is below the other.  A draw then is the number of borders that
// are not above u, and rows of many draws are bound by memory: 200,000 rows of 8 places with 1,024 draws each read and write
// 1.03 GB in 222 us, 4.6 TB/s.
template <typename T, int L, int PER, typename TT>
__global__ __launch_bounds__(kFewThreads) void few_sample_kernel(Draw d) {
    constexpr int kRowsHere = kFewThreads / L, kPer = PER, kRoom = L * kPer;
    __shared__ float border[kRowsHere][kRoom + 1], lp[kRowsHere][kRoom + 1], xs[kRowsHere][kRoom + 1];
    __shared__ double ps[kRowsHere][kRoom];
    __shared__ bool empty[kRowsHere];
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
    for (int i = 0; i < kPer; i++) p[i] = none || x[i] == -INFINITY ? 0.0 : power_of_two(((double)x[i] - (double)m) * rule.scale * kLog2eWide);
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
    if (lane == 0) empty[mine] = none;
    __syncthreads();
    // The draws: a wavefront a row where a row has many, else one after the other
    const int64_t row0 = (int64_t)group_number() * kRowsHere;
    const int rows = (int)min((int64_t)kRowsHere, max(d.rows - row0, (int64_t)0));      // (none of a grid's last row that are too many)
    if (d.given >= kWave) {
        const int wlane = threadIdx.x % kWave;
        for (int r = threadIdx.x / kWave; r < rows; r += kFewThreads / kWave) draw_row<TT>(d, row0 + r, border[r], lp[r], empty[r], wlane, kWave);
    } else {
        const int all = rows * d.given;
        for (int i = threadIdx.x; i < all; i += kFewThreads) {
            const int r = i / d.given;
            draw_row<TT>(d, row0 + r, border[r], lp[r], empty[r], i % d.given, INT32_MAX / 2);
        }
    }
}

// ---- rows of many places -----------------------------------------------------------------------------

constexpr int kChunks = 2048;                // of a row, whose masses are kept
constexpr int kBins = 2048, kCopies = 2;     // of the digits of a key; lanes that meet in a bin go to copies
constexpr int kSteps = 256, kLanes = 16;     // of mass by depth below the best; as many copies
constexpr int kListed = 2048;                // places that a list has room for
constexpr int kRanked = 512;                 // up to which a list is put in order by counting
static_assert(kBins * kCopies == kSteps * kLanes);

template <int THREADS>
struct Block {
    static constexpr int kWaves = THREADS / kWave;
    union {
        float f[kWaves];
        uint64_t u[kWaves];
        double d[kWaves];
        int32_t i[kWaves];
    };
    __device__ __forceinline__ float *of(float) { return f; }
    __device__ __forceinline__ uint64_t *of(uint64_t) { return u; }
    __device__ __forceinline__ double *of(double) { return d; }
    __device__ __forceinline__ int32_t *of(int32_t) { return i; }

    // the sum over the threads in front of one's own; total of all
    template <typename N>
    __device__ __forceinline__ N before(N v, N &total) {
        const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
        N upto = v;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const N o = __shfl_up(upto, off);
            if (lane >= off) upto += o;
        }
        N *room = of(N{});
        __syncthreads();
        if (lane == kWave - 1) room[wave] = upto;
        __syncthreads();
        N front = 0;
        total = 0;
#pragma unroll
        for (int w = 0; w < kWaves; w++) {
            if (w < wave) front += room[w];
            total += room[w];
        }
        return front + upto - v;
    }
};

// The words of a list from the largest on.  Few are counted into their places, more go through a sorting network.
template <int THREADS>
__device__ __forceinline__ void put_in_order(uint64_t *list, int count) {
    if (count <= kRanked) {
        constexpr int kOwn = (kRanked + THREADS - 1) / THREADS;
        uint64_t own[kOwn];
        int rank[kOwn];
#pragma unroll
        for (int o = 0; o < kOwn; o++) {
            const int i = threadIdx.x + o * THREADS;
            own[o] = i < count ? list[i] : 0, rank[o] = 0;
        }
        if (count > (int)(threadIdx.x & ~(kWave - 1)))         // (a wavefront with words)
            for (int k = 0; k < count; k++) {
                const uint64_t other = list[k];
#pragma unroll
                for (int o = 0; o < kOwn; o++) rank[o] += other > own[o];
            }
        __syncthreads();
#pragma unroll
        for (int o = 0; o < kOwn; o++)
            if ((int)threadIdx.x + o * THREADS < count) list[rank[o]] = own[o];
        __syncthreads();
        return;
    }
    int size = 2;
    while (size < count) size *= 2;
    for (int i = count + (int)threadIdx.x; i < size; i += THREADS) list[i] = 0;
    __syncthreads();
    for (int run = 2; run <= size; run *= 2)
        for (int step = run / 2; step > 0; step /= 2) {
            for (int k = threadIdx.x; k < size / 2; k += THREADS) {
                const int i = 2 * k - (k & (step - 1)), j = i + step;
                const uint64_t a = list[i], b = list[j];
                if ((a < b) == ((i & run) == 0)) list[i] = b, list[j] = a;
            }
            __syncthreads();
        }
}

// A workgroup a row, which is read from the caches for each of: the maximum; where what is kept ends; the mass of each chunk; the draws.  Only
// the first reads it from memory.  512 of 65,536 with settings of their own 174 to 187 us.  These are bound by the probabilities (some 16 operations of
// 64 bits each) and by the sums of mass by depth, an atomic operation of 64 bits a place in LDS (about 55 us of a row's time).
template <typename T, int THREADS>
struct Many {
    static constexpr int kVec = 16 / (int)sizeof(T), kStep = kWave * kVec;      // places of a lane and of a wavefront's load
    static constexpr int kLevels = sizeof(T) == 2 ? 2 : 3, kDrop = sizeof(T) == 2 ? 10 : 0;        // digits of 11, 11 and 10 bits

    const T *row;
    const uint64_t *allow;
    int32_t V;
    float m;
    double scale;                        // (of exponents of 2)

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
    // f(place, its logit) for all places, the workgroup's threads side by side, with AHEAD vectors a thread under way at once
    template <int AHEAD, typename F>
    __device__ __forceinline__ void each(F f) const {
        constexpr int kSide = THREADS * kVec;
        int32_t v = threadIdx.x * kVec;
        const int32_t whole = V / (kSide * AHEAD) * (kSide * AHEAD);
        for (; v < whole; v += kSide * AHEAD) {
            Pack<T, kVec> at[AHEAD];
            uint64_t bits[AHEAD];
#pragma unroll
            for (int q = 0; q < AHEAD; q++) at[q] = load_pack<T, kVec>(row + v + q * kSide);
#pragma unroll
            for (int q = 0; q < AHEAD; q++) bits[q] = allow ? allow[(v + q * kSide) >> 6] >> (v & 63) : ~0ull;      // (64 divides kSide)
#pragma unroll
            for (int q = 0; q < AHEAD; q++)
#pragma unroll
                for (int i = 0; i < kVec; i++) f(v + q * kSide + i, bits[q] >> i & 1 ? (float)at[q].v[i] : -INFINITY);
        }
        for (; v < V; v += kSide) {
            float x[kVec];
            load(v, x);
#pragma unroll
            for (int i = 0; i < kVec; i++)
                if (v + i < V) f(v + i, x[i]);
        }
    }
    __device__ __forceinline__ double depth(float x) const { return ((double)m - (double)x) * scale; }
    __device__ __forceinline__ double share(float x) const { return x == -INFINITY ? 0.0 : power_of_two(-depth(x)); }
    __device__ __forceinline__ static uint32_t key(float x) { return order_key(x) >> kDrop; }
    __device__ __forceinline__ static float value(uint32_t key) {
        uint32_t b = key << kDrop;
        if (b & 0x80000000u) b &= 0x7fffffffu;
        else b = ~(b | ((1u << kDrop) - 1));
        return __uint_as_float(b);
    }
    __device__ __forceinline__ static int shift(int level) { return kLevels == 2 ? 11 - 11 * level : 21 - 11 * level + (level == 2); }
};

__device__ __forceinline__ uint64_t listed(uint32_t key, int32_t place) { return (uint64_t)key << 32 | (0xffffffffu - (uint32_t)place); }

// Lists the best top_k <= THREADS places and a few more, those of places from `from` on; their number, which may be more than there is room for.
// The bound that they are at or above is the least of what a few threads' own best places of each wavefront reach; a thread has few of a row's
// best.  (own, m: of the thread and of all.)
template <typename T, int THREADS>
__device__ __forceinline__ int list_best(const Many<T, THREADS> &a, float own, float m, int32_t top_k, int32_t from, uint64_t *list, Block<THREADS> &block, int &counted_) {
    using M = Many<T, THREADS>;
    constexpr int kWaves = THREADS / kWave;
    const int share = (top_k + kWaves - 1) / kWaves;
    const uint32_t key = M::key(own);
    uint32_t low = 0, high = M::key(m) + 1;
    for (int n = 0; n < 32 && high - low > 1; n++) {
        const uint32_t mid = low + (high - low) / 2;
        if (__popcll(__ballot(key >= mid)) >= share) low = mid;
        else high = mid;
    }
    if (threadIdx.x % kWave == 0) block.i[threadIdx.x / kWave] = (int32_t)(low ^ 0x80000000u);
    if (threadIdx.x == 0) counted_ = 0;
    __syncthreads();
    int32_t least = block.i[0];
#pragma unroll
    for (int w = 1; w < kWaves; w++) least = min(least, block.i[w]);
    low = (uint32_t)least ^ 0x80000000u;
    a.template each<4>([&](int32_t v, float x) {
        if (M::key(x) >= low && x > -INFINITY) {
            const int at = atomicAdd(&counted_, 1);
            if (at < kListed) list[at] = listed(M::key(x), from + v);
        }
    });
    __syncthreads();
    const int count = counted_;
    __syncthreads();
    return count;
}

// Few long rows of which few places are kept: a workgroup a slice of a row lists the slice's best top_k, and many_sample_kernel begins with these.
constexpr int kSliced = 128, kSlices = 64;   // top_k, and slices of a row, at most
constexpr int32_t kSlice = 8192;             // places of a slice at least
constexpr int kSliceThreads = 256;
constexpr int32_t kNoRoom = -1, kOdd = -2;
__device__ __forceinline__ bool sliced(const Draw &d, const Rule &r) { return d.slices > 0 && r.fine && r.top_k > 0 && r.top_k <= kSliced; }
// (top_p of 0: the best alone)
__device__ __forceinline__ Rule row_rule(const Draw &d, int64_t row) {
    Rule r = rule_of(d.set, row);
    if (r.top_p == 0.0) r.top_p = 1.0, r.top_k = 1;
    if (r.top_k >= d.vocab) r.top_k = 0;
    return r;
}

template <typename T>
__global__ __launch_bounds__(kSliceThreads) void slice_list_kernel(Draw d) {
    using M = Many<T, kSliceThreads>;
    __shared__ uint64_t list[kListed];
    __shared__ Block<kSliceThreads> block;
    __shared__ int odd_, counted_;
    const uint32_t group = group_number();
    const int64_t row = group / d.slices;
    if (row >= d.rows) return;
    const Rule rule = row_rule(d, row);
    if (!sliced(d, rule)) return;
    const int32_t from = (int32_t)(group % d.slices) * d.slice_size;
    const M a{(const T *)d.logits + row * d.ld + from, d.allow ? d.allow + row * d.words + from / 64 : nullptr, min(d.slice_size, d.vocab - from), 0.0f, 0.0};
    if (threadIdx.x == 0) odd_ = 0;
    float own = -INFINITY;
    bool odd = false;
    a.template each<4>([&](int32_t, float x) { odd |= !(x < INFINITY), own = fmaxf(own, x); });
    float m = most_of<kWave>(own);
    if (threadIdx.x % kWave == 0) block.f[threadIdx.x / kWave] = m;
    __syncthreads();
    if (odd) odd_ = 1;
#pragma unroll
    for (int w = 0; w < kSliceThreads / kWave; w++) m = fmaxf(m, block.f[w]);
    __syncthreads();
    int32_t found = kOdd;
    if (!odd_) {
        const int count = list_best<T, kSliceThreads>(a, own, m, rule.top_k, from, list, block, counted_);
        found = kNoRoom;
        if (count <= kListed) {
            put_in_order<kSliceThreads>(list, count);
            found = min(count, rule.top_k);
            if ((int)threadIdx.x < found) d.found[(int64_t)group * kSliced + threadIdx.x] = list[threadIdx.x];
        }
    }
    if (threadIdx.x == 0) d.counts[group] = found;
}

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == 256 ? 2 : 4) void many_sample_kernel(Draw d) {
    using M = Many<T, THREADS>;
    constexpr int kVec = M::kVec, kStep = M::kStep, kWaves = THREADS / kWave;
    __shared__ uint64_t bins[kBins * kCopies], list[kListed];
    __shared__ double mass[kChunks];
    __shared__ int32_t ties[kChunks];
    __shared__ Block<THREADS> block;
    __shared__ int odd_, found_at, counted_;
    __shared__ uint64_t found_above;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t row = group_number();
    if (row >= d.rows) return;
    const Rule rule = row_rule(d, row);
    const int32_t V = d.vocab;
    M a{(const T *)d.logits + row * d.ld, d.allow ? d.allow + row * d.words : nullptr, V, 0.0f, rule.scale * kLog2eWide};
    const auto draw_of = [&](int32_t g) { return (double)counted(d.u[row * d.u_row + g * d.u_step]); };
    const auto put_logp = [&](int32_t g, float x, double logs) {
        if (d.logp) d.logp[row * d.given + g] = (float)(((double)x - (double)a.m) * rule.scale - logs);
    };

    if (threadIdx.x == 0) odd_ = counted_ = 0;
    __syncthreads();
    float own = -INFINITY, m = -INFINITY;
    int32_t have = INT_MAX;                            // words in the list
    bool whole = true;                                 // whether the row is to be read
    if (sliced(d, rule)) {
        // The slices' lists: of each the first words, as many as make top_k together, are at or above a bound
        const uint64_t *from = d.found + row * d.slices * kSliced;
        const int32_t *counts = d.counts + row * d.slices;
        const int32_t mine = lane < d.slices ? counts[lane] : 0, share = (rule.top_k + d.slices - 1) / d.slices;
        uint64_t bound = lane >= d.slices ? ~0ull : mine >= share ? from[lane * kSliced + share - 1] : 0, best = mine > 0 ? from[lane * kSliced] : 0;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            bound = min(bound, (uint64_t)__shfl_xor((unsigned long long)bound, off));
            best = max(best, (uint64_t)__shfl_xor((unsigned long long)best, off));
        }
        if (__ballot(mine == kOdd)) odd_ = 1, whole = false;
        else if (!__ballot(mine == kNoRoom)) {
            whole = false;
            m = best ? M::value((uint32_t)(best >> 32)) : -INFINITY;
            for (int i = threadIdx.x; i < d.slices * rule.top_k; i += THREADS) {
                const int s = i / rule.top_k, k = i - s * rule.top_k;
                const uint64_t word = k < counts[s] ? from[s * kSliced + k] : 0;
                if (word && word >= bound) {
                    const int at = atomicAdd(&counted_, 1);
                    if (at < kListed) list[at] = word;
                }
            }
        }
        __syncthreads();
        have = counted_;
        if (!whole && have > kListed) whole = true;
        __syncthreads();
        if (threadIdx.x == 0) counted_ = 0;
    }
    if (whole) {
        have = INT_MAX;
        bool odd = false;
        a.template each<4>([&](int32_t, float x) { odd |= !(x < INFINITY), own = fmaxf(own, x); });
        m = most_of<kWave>(own);
        if (lane == 0) block.f[wave] = m;
        __syncthreads();
        if (odd) odd_ = 1;
#pragma unroll
        for (int w = 0; w < kWaves; w++) m = fmaxf(m, block.f[w]);
    }
    a.m = m;
    __syncthreads();
    if (odd_ || m == -INFINITY || !rule.fine) {
        if (!rule.fine && threadIdx.x == 0) atomicOr(d.status, CP_STATUS_BAD_SAMPLING);
        for (int32_t g = threadIdx.x; g < d.given; g += THREADS) {
            put_token(d, row, g, -1);
            if (d.logp) d.logp[row * d.given + g] = 0.0f;
        }
        return;
    }
    // adds a place to the list, if there is room
    const auto note = [&](float x, int32_t v) {
        const int at = atomicAdd(&counted_, 1);
        if (at < kListed) list[at] = listed(M::key(x), v);
    };

    // Few are left: they are listed, put in order, and all the rest is a matter of the list.
    if (rule.top_k > 0 && rule.top_k <= THREADS) {
        const int count = have != INT_MAX ? have : list_best<T, THREADS>(a, own, m, rule.top_k, 0, list, block, counted_);
        if (threadIdx.x == 0) counted_ = 0;
        if (count <= kListed) {
            put_in_order<THREADS>(list, count);
            // by rank: shares, what lies in front, what is kept (the first ones)
            const int n = min(count, rule.top_k), i = threadIdx.x;
            const uint64_t one = i < n ? list[i] : 0;
            const double p = i < n ? a.share(M::value((uint32_t)(one >> 32))) : 0.0;
            double total;
            const double ahead = block.before(p, total);
            const bool keep = i < n && (i == 0 || rule.top_p >= 1.0 || ahead < rule.top_p * total) && p >= rule.min_p;
            const int kept = __syncthreads_count(keep);
            // and by place
            if (keep) list[i] = (uint64_t)(uint32_t)one << 32 | (uint32_t)(one >> 32);
            __syncthreads();
            put_in_order<THREADS>(list, kept);
            const double q = i < kept ? a.share(M::value((uint32_t)list[i])) : 0.0;
            double all;
            const double before = block.before(q, all);
            if (i < kept) mass[i] = before + q;
            __syncthreads();
            for (int32_t g = threadIdx.x; g < d.given; g += THREADS) {
                const double target = draw_of(g) * all;
                int lo = 0, hi = kept - 1;
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    if (mass[mid] > target) hi = mid;
                    else lo = mid + 1;
                }
                put_token(d, row, g, (int32_t)(0xffffffffu - (uint32_t)(list[lo] >> 32)));
                put_logp(g, M::value((uint32_t)list[lo]), d.logp ? log(all) : 0.0);
            }
            return;
        }
    }

    // The place in the order where what is kept ends: keys above `key_end`, and `keep_ties` of those that equal it
    uint32_t key_end = 0;
    int64_t keep_ties = INT64_MAX;
    // Masses are added up as whole numbers, which come to the same in any order: those of a step or a digit in units that its sum has just room
    // for, and these sums in units of 2^-61 to 2^-62 of the whole row's.
    const auto scale_of = [](double total) { return ldexp(1.0, 61 - ilogb(total)); };
    const auto in_units = [](double mass, double scale) { return (uint64_t)(mass * scale + 0.5); };
    if (rule.top_p < 1.0 && rule.top_k == 0) {
        // By how far places lie below the best: 240 steps of a twelfth of a power of two and 16 of one, the step in which top_p is reached again in 256, and so
        // on until the places of a step are few, which are listed and put in order.  A step's unit is 2^-bits of the mass of a place at its beginning, or
        // of up to twice that, of which all its places have at least a quarter.  So a row's masses are off by 2^(1 - bits) of themselves, 3e-14 in rows of
        // 2^20 places and 2e-12 in such of 2^26, however flat they are.  (With one unit for all steps 2e-7 and 1e-3; 512 x 65536 with settings of their own
        // 180 us; 187 with one a step.)
        constexpr int kDepth = 6, kFine = 240, kPer = 12, kRest = kFine - kFine / kPer;      // (wide steps: powers + kRest)
        const int bits = 63 - (32 - __clz(min(V, V / kLanes + THREADS * kVec / kLanes)));      // (of a copy's lanes together, below 2^64)
        __shared__ double from[kDepth + 1], per[kDepth + 1];
        __shared__ int at[kDepth + 1];
        uint64_t above = 0;
        double want = 0, scale = 0;
        const auto twelfths = [](int i) { return (int)(__umul24(i, 171) >> 11); };      // i / 12 below 512
        const auto step_of = [&](double depth, int level) {
            if (level > 0) return (int)fmin(fmax((depth - from[level]) * per[level], 0.0), kSteps - 1.0);
            const int i = (int)fmin(depth * kPer, (kSteps - kRest) * kPer - 1.0);
            return i < kFine ? i : twelfths(i) + kRest;
        };
        // whole powers of two that a step begins below the best, or the step that it is part of
        const auto powers_of = [&](int step, int level) { return level > 0 ? (int)from[level] : step < kFine ? twelfths(step) : step - kRest; };
        const auto inside = [&](double depth, int level) {     // whether it lies in the step of all levels before this one
            bool in = true;
            for (int k = 0; k < level; k++) in &= step_of(depth, k) == at[k];
            return in;
        };
        for (int level = 0; level < kDepth && keep_ties == INT64_MAX; level++) {
            for (int i = threadIdx.x; i < kSteps * kLanes; i += THREADS) bins[i] = 0;
            if (threadIdx.x == 0) counted_ = 0;
            __syncthreads();
            a.template each<2>([&](int32_t v, float x) {
                const double depth = a.depth(x);
                if (x > -INFINITY && inside(depth, level)) {
                    const int step = step_of(depth, level);
                    atomicAdd((unsigned long long *)&bins[step * kLanes + lane % kLanes],
                              (unsigned long long)(power_of_two(-depth, bits + powers_of(step, level)) + 0.5));
                    if (level > 0) note(x, v);
                }
            });
            __syncthreads();
            const int count = level > 0 ? counted_ : INT_MAX;          // (read here: it is cleared behind the barriers below)
            // (thread t has steps 256 / THREADS t and on)
            constexpr int kEach = THREADS < kSteps ? kSteps / THREADS : 1;
            uint64_t sum = 0, one[kEach];
            double held[kEach], all = 0;
#pragma unroll
            for (int e = 0; e < kEach; e++) {
                held[e] = 0;
                const int step = (int)threadIdx.x * kEach + e;
                if (step < kSteps) {
                    for (int k = 0; k < kLanes; k++) held[e] += (double)bins[step * kLanes + k];
                    held[e] = ldexp(held[e], -bits - powers_of(step, level));
                }
                all += held[e];
            }
            if (level == 0) {
                double row_mass;
                block.before(all, row_mass);
                scale = scale_of(row_mass);
            }
#pragma unroll
            for (int e = 0; e < kEach; e++) sum += one[e] = in_units(held[e], scale);
            uint64_t total;
            uint64_t front = above + block.before(sum, total);
            if (level == 0) want = (double)total * rule.top_p;
            if (threadIdx.x == 0) found_at = kSteps - 1, found_above = above + total;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kEach; e++) {
                const int step = (int)threadIdx.x * kEach + e;
                if (step < kSteps && (double)front < want && !((double)(front + one[e]) < want)) found_at = step, found_above = front;
                front += one[e];
            }
            __syncthreads();
            const int step = found_at;
            above = found_above;
            if (threadIdx.x == 0) {
                at[level] = step;
                if (level == 0) {
                    from[1] = step < kFine ? (double)step / kPer : step - kRest;
                    per[1] = kSteps * (step < kFine ? kPer : step < kSteps - 1 ? 1.0 : 1 / 1100.0);
                } else {
                    from[level + 1] = from[level] + step / per[level];
                    per[level + 1] = per[level] * kSteps;
                }
                counted_ = 0;
            }
            __syncthreads();
            if (count > kListed) continue;
            // those of the list that lie in the step
            constexpr int kOwn = (kListed + THREADS - 1) / THREADS;
            uint64_t mine[kOwn];
#pragma unroll
            for (int o = 0; o < kOwn; o++) mine[o] = (int)threadIdx.x + o * THREADS < count ? list[threadIdx.x + o * THREADS] : 0;
            __syncthreads();
#pragma unroll
            for (int o = 0; o < kOwn; o++)
                if (mine[o] && step_of(a.depth(M::value((uint32_t)(mine[o] >> 32))), level) == step) list[atomicAdd(&counted_, 1)] = mine[o];
            __syncthreads();
            const int few = counted_;
            if (few == 0) continue;                    // (a rounding of `want`)
            put_in_order<THREADS>(list, few);
            int kept = 0;
            for (int i0 = 0; i0 < few; i0 += THREADS) {
                const int i = i0 + threadIdx.x;
                const uint64_t w = i < few ? in_units(a.share(M::value((uint32_t)(list[i] >> 32))), scale) : 0;
                uint64_t all;
                const uint64_t ahead = above + block.before(w, all);
                kept += __syncthreads_count(i < few && (i == 0 || (double)ahead < want));
                above += all;
            }
            key_end = (uint32_t)(list[kept - 1] >> 32);
            keep_ties = 0;
            for (int i0 = 0; i0 < kept; i0 += THREADS)
                keep_ties += __syncthreads_count(i0 + (int)threadIdx.x < kept && (uint32_t)(list[min(i0 + (int)threadIdx.x, kListed - 1)] >> 32) == key_end);
        }
    }
    if (keep_ties == INT64_MAX && (rule.top_k > 0 || rule.top_p < 1.0)) {
        // Many, or all alike: by the digits of their keys, from the highest on, first as many as top_k, then as much as top_p
        const auto count_in = [&](int i) { return bins[i] + bins[kBins + i]; };
        const auto seek = [&](auto bin, double want, uint64_t above) {
            // (thread t has the t-th few bins from the top)
            constexpr int kEach = kBins / THREADS;
            uint64_t one[kEach], sum = 0, total;
#pragma unroll
            for (int e = 0; e < kEach; e++) sum += one[e] = bin(kBins - 1 - kEach * (int)threadIdx.x - e);
            uint64_t front = above + block.before(sum, total);
            if (threadIdx.x == 0) found_at = 0, found_above = above + total;       // (rounding: the lowest)
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kEach; e++) {
                if ((double)front < want && !((double)(front + one[e]) < want)) found_at = kBins - 1 - kEach * (int)threadIdx.x - e, found_above = front;
                front += one[e];
            }
            __syncthreads();
        };
        const auto clear = [&] {
            __syncthreads();
            for (int i = threadIdx.x; i < kBins * kCopies; i += THREADS) bins[i] = 0;
            __syncthreads();
        };
        if (rule.top_k > 0) {
            uint64_t above = 0;
            uint32_t prefix = 0;
            for (int level = 0; level < M::kLevels; level++) {
                const int sh = M::shift(level), width = level == 2 ? 10 : 11;
                clear();
                a.template each<2>([&](int32_t, float x) {
                    const uint32_t k = M::key(x);
                    if (level == 0 || k >> (sh + width) == prefix) atomicAdd((unsigned int *)&bins[lane % kCopies * kBins + (k >> sh & ((1u << width) - 1))], 1u);
                });
                __syncthreads();
                seek(count_in, (double)rule.top_k, above);
                prefix = prefix << width | (uint32_t)found_at, above = found_above;
            }
            key_end = prefix, keep_ties = (int64_t)rule.top_k - (int64_t)above;
        }
        if (rule.top_p < 1.0) {
            const uint32_t least = key_end;
            const int64_t least_ties = keep_ties;
            // masses in two words: the places of a digit may be of any, so that one has too few bits for rows whose most lies in many unlikely places
            const int bits = 63 - (32 - __clz(V));
            const auto add = [&](int at, double mass) {
                const double units = ldexp(mass, bits), whole = floor(units);
                atomicAdd((unsigned long long *)&bins[at], (unsigned long long)whole);
                atomicAdd((unsigned long long *)&bins[kBins + at], (unsigned long long)(ldexp(units - whole, bits) + 0.5));
            };
            const auto mass_in = [&](int i) { return ldexp((double)bins[i] + ldexp((double)bins[kBins + i], -bits), -bits); };
            uint64_t above = 0;
            uint32_t prefix = 0;
            double want = 0, scale = 0;
            for (int level = 0; level < M::kLevels; level++) {
                const int sh = M::shift(level), width = level == 2 ? 10 : 11;
                clear();
                a.template each<1>([&](int32_t, float x) {
                    const uint32_t k = M::key(x);
                    // (of those that equal the last of the top_k, added below, only some are left)
                    if (x > -INFINITY && (k > least || least_ties == INT64_MAX) && (level == 0 || k >> (sh + width) == prefix))
                        add(k >> sh & ((1u << width) - 1), a.share(x));
                });
                __syncthreads();
                if (threadIdx.x == 0 && least_ties != INT64_MAX && (level == 0 || least >> (sh + width) == prefix))
                    add(least >> sh & ((1u << width) - 1), (double)least_ties * a.share(M::value(least)));
                __syncthreads();
                const auto units_in = [&](int i) { return in_units(mass_in(i), scale); };
                if (level == 0) {
                    double sum = 0, row_mass;
                    for (int i = threadIdx.x; i < kBins; i += THREADS) sum += mass_in(i);
                    block.before(sum, row_mass);
                    scale = scale_of(row_mass);
                    uint64_t units = 0, total;
                    for (int i = threadIdx.x; i < kBins; i += THREADS) units += units_in(i);
                    block.before(units, total);
                    want = (double)total * rule.top_p;
                }
                seek(units_in, want, above);
                prefix = prefix << width | (uint32_t)found_at, above = found_above;
            }
            // places that equal the last one: as long as less than `want` lies in front of them, the first in any case
            const double each = a.share(M::value(prefix)) * scale, front = (double)above;
            int64_t more = V;
            if (each > 0) {
                more = (int64_t)fmin(fmax((want - front) / each, 0.0), (double)V);
                while (more > 0 && !(front + (double)(more - 1) * each < want)) more--;
                while (more < V && front + (double)more * each < want) more++;
            }
            more = max(more, (int64_t)(above == 0));
            if (prefix == least) more = min(more, least_ties);
            key_end = prefix, keep_ties = more;
        }
    }
    // what equals the last one and is less likely than min_p goes too
    const double end_share = keep_ties == INT64_MAX ? 0.0 : a.share(M::value(key_end));
    if (keep_ties != INT64_MAX && end_share < rule.min_p) keep_ties = 0;
    const bool cut = keep_ties != INT64_MAX;

    // The row in chunks, one after the other: mass above the end, and how many equal it
    const int32_t steps = (int32_t)(((int64_t)V + (int64_t)kStep * kChunks - 1) / ((int64_t)kStep * kChunks));       // of a chunk
    const int64_t size = (int64_t)steps * kStep;
    const int32_t chunks = (int32_t)((V + size - 1) / size);
    const auto kept = [&](float x, bool &tie) {
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
    constexpr int kAtOnce = 2;                         // chunks of a wavefront under way at once
    for (int32_t first = wave * kAtOnce; first < chunks; first += kWaves * kAtOnce) {
        double sum[kAtOnce] = {};
        int32_t same[kAtOnce] = {};
        for (int32_t s = 0; s < steps; s++) {
            float x[kAtOnce][kVec];
#pragma unroll
            for (int q = 0; q < kAtOnce; q++) a.load((int32_t)min((first + q) * size + s * kStep + lane * kVec, (int64_t)V), x[q]);
#pragma unroll
            for (int q = 0; q < kAtOnce; q++)
#pragma unroll
                for (int i = 0; i < kVec; i++) {
                    bool tie;
                    sum[q] += kept(x[q][i], tie);
                    same[q] += tie;
                }
        }
#pragma unroll
        for (int q = 0; q < kAtOnce; q++) {
            sum[q] = sum_of<kWave>(sum[q]);
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) same[q] += __shfl_xor(same[q], off);
            if (lane == 0 && first + q < chunks) mass[first + q] = sum[q], ties[first + q] = same[q];
        }
    }
    __syncthreads();
    // masses up to and with each chunk, and ties in front of it, of which the first ones by place are kept
    double total = 0;
    {
        constexpr int kEach = kChunks / THREADS;
        const int32_t c0 = kEach * threadIdx.x;
        int32_t own_ties[kEach], sum_ties = 0, all_ties;
        double own_mass[kEach], sum_mass = 0;
#pragma unroll
        for (int e = 0; e < kEach; e++) sum_ties += own_ties[e] = c0 + e < chunks ? ties[c0 + e] : 0;
        int64_t front = block.before(sum_ties, all_ties);
#pragma unroll
        for (int e = 0; e < kEach; e++) {
            own_mass[e] = c0 + e < chunks ? mass[c0 + e] : 0;
            if (cut) own_mass[e] += (double)max(min((int64_t)own_ties[e], keep_ties - front), (int64_t)0) * end_share;
            if (c0 + e < chunks) ties[c0 + e] = (int32_t)front;
            front += own_ties[e];
            sum_mass += own_mass[e];
        }
        double upto = block.before(sum_mass, total);
#pragma unroll
        for (int e = 0; e < kEach; e++) {
            upto += own_mass[e];
            if (c0 + e < chunks) mass[c0 + e] = upto;
        }
    }
    __syncthreads();
    const double logs = d.logp ? log(total) : 0.0;

    for (int32_t g = wave; g < d.given; g += kWaves) {
        const double target = draw_of(g) * total;
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
                    double here = before + upto;
#pragma unroll
                    for (int i = kVec - 1; i >= 0; i--) {
                        // (from the back: the first place that reaches beyond is the last one seen; the lane's last place in any case)
                        if (p[i] > 0 && here > target) hit = (int32_t)v + i;
                        here -= p[i];
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
            put_logp(g, (float)a.row[max(token, 0)], logs);
        }
    }
}

constexpr int64_t kFar = 1ll << 28;          // strides; products of these, rows and bytes stay in 64 bits

// Slices of a row, or 0 where rows are not cut: more rows fill the chip by themselves, and shorter ones are done before a second launch begins.  (bf16,
// top_k 50 and top_p 0.9: 8 x 131072 23 us, 34 uncut; 64 x 131072 29, 35; 8 x 524288 30, 88; but 8 x 32768 21.4, 19.4.  top_k 128: 8 x 131072 30 us, 37;
// 256, whose lists are long, 93, 43.)
int32_t slice_size_of(int32_t vocab) { return (int32_t)std::max<int64_t>(((int64_t)vocab + (int64_t)kSlices * kSlice - 1) / ((int64_t)kSlices * kSlice), 1) * kSlice; }
int32_t slices_of(int64_t rows, int32_t vocab) {
    if (rows < 1 || rows > 64 || vocab < 8 * kSlice) return 0;
    return (vocab + slice_size_of(vocab) - 1) / slice_size_of(vocab);
}
size_t found_bytes(int64_t rows, int32_t slices) { return align_up((size_t)rows * slices * kSliced * sizeof(uint64_t)); }

__global__ void clear_sampling_kernel(int32_t *status) { *status = CP_STATUS_OK; }

}  // namespace

}  // namespace cpeval

using namespace cpeval;

extern "C" {

int cp_token_sample_workspace_bytes(int64_t rows, int32_t vocab, int32_t given, size_t *out_bytes) {
    if (!out_bytes) return CP_ERR_NULL;
    if (rows < 0 || rows > INT32_MAX || vocab < 1 || vocab > CP_LOGPROBS_MAX_VOCAB || given < 0 || given > CP_LOGPROBS_MAX_GIVEN) return CP_ERR_SIZE;
    const int32_t slices = given > 0 ? slices_of(rows, vocab) : 0;
    *out_bytes = slices ? found_bytes(rows, slices) + align_up((size_t)rows * slices * sizeof(int32_t)) : 0;
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
    if (need) {
        if (!workspace) return CP_ERR_NULL;
        if ((uintptr_t)workspace % kPolicyAlign || workspace_bytes < need) return CP_ERR_WORKSPACE;
    }
    // (what there is one of is at no distance from another)
    if (rows == 1) u_row_stride = token_row_stride = 0;
    if (given == 1) u_stride = token_stride = 0;
    if (rows > 0 && given > 0) {
        // numbers may lie anywhere, tokens apart from each other
        if (u_row_stride < 0 || u_stride < 0 || u_row_stride > kFar || u_stride > kFar || token_row_stride > kFar || token_stride > kFar) return CP_ERR_SIZE;
        const bool apart = token_row_stride >= (given - 1) * token_stride + 1, between = token_stride >= (rows - 1) * token_row_stride + 1;
        if ((given > 1 && token_stride < 1) || (rows > 1 && token_row_stride < 1) || (given > 1 && rows > 1 && !apart && !between)) return CP_ERR_SIZE;
        const int64_t each = token_type, t_row = token_row_stride, t_step = token_stride;
        const Extent to = rows == 1   ? Extent{tokens, 1, ((given - 1) * t_step + 1) * each, 0, (size_t)each}
                          : given == 1 || apart ? Extent{tokens, rows, ((given - 1) * t_step + 1) * each, t_row * each, (size_t)each}
                                                : Extent{tokens, given, ((rows - 1) * t_row + 1) * each, t_step * each, (size_t)each};
        const Extent numbers = vector_at(u, (rows - 1) * u_row_stride + (given - 1) * u_stride + 1);
        if (in_the_way({matrix_at(logits, rows, vocab, ld, type), numbers, vector_at(allow, rows * ((vocab + 63) / 64), 8), vector_at(scales, rows),
                        vector_at(top_ks, rows), vector_at(top_ps, rows), vector_at(min_ps, rows)},
                       {to, vector_at(logp, rows * given), vector_at(own ? status_out : nullptr, 1), vector_at(need ? workspace : nullptr, (int64_t)need, 1)}))
            return CP_ERR_ARG;
    }
    const hipStream_t st = (hipStream_t)stream;
    if (own) hipLaunchKernelGGL(clear_sampling_kernel, dim3(1), dim3(1), 0, st, status_out);
    if (rows == 0 || given == 0) return launched();
    // (only where a row may keep few places; not for the sake of a row's own top_p of 0)
    const int32_t slices = top_ks || (top_k > 0 && top_k <= kSliced) || (!top_ps && top_p == 0.0) ? slices_of(rows, vocab) : 0;
    const Draw d{rows, vocab, (vocab + 63) / 64, logits, ld, allow, {scale, top_p, min_p, top_k, scales, top_ps, min_ps, top_ks}, given, u,
                 u_row_stride, u_stride, tokens, token_type, token_row_stride, token_stride, logp, status_out, slices, slice_size_of(vocab),
                 (uint64_t *)workspace, (int32_t *)((char *)workspace + (slices ? found_bytes(rows, slices) : 0))};
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        if (vocab > kFew) {
            if (slices) {
                hipLaunchKernelGGL((slice_list_kernel<T>), grid_of(rows * slices), dim3(kSliceThreads), 0, st, d);
                const int code = launched();
                if (code) return code;
            }
            // A workgroup as large as has work for its threads (2048 x 4000 bf16 46 us, 85 of 1,024 threads), two a compute unit where there are more
            // rows than compute units (512 x 65536 187 us, 191 of 1,024 threads; but 8 x 131072 34 us, 36 of 512).
            if (vocab <= 8192) hipLaunchKernelGGL((many_sample_kernel<T, 256>), grid_of(rows), dim3(256), 0, st, d);
            else if (rows > 256) hipLaunchKernelGGL((many_sample_kernel<T, 512>), grid_of(rows), dim3(512), 0, st, d);
            else hipLaunchKernelGGL((many_sample_kernel<T, 1024>), grid_of(rows), dim3(1024), 0, st, d);
            return launched();
        }
        auto go = [&](auto l, auto each) {
            constexpr int L = decltype(l)::value, PER = decltype(each)::value;
            auto *kernel = token_type == CP_TOKEN_U8    ? few_sample_kernel<T, L, PER, uint8_t>
                           : token_type == CP_TOKEN_I32 ? few_sample_kernel<T, L, PER, int32_t>
                                                        : few_sample_kernel<T, L, PER, int64_t>;
            hipLaunchKernelGGL(kernel, grid_of((rows + kFewThreads / L - 1) / (kFewThreads / L)), dim3(kFewThreads), 0, st, d);
            return launched();
        };
        const std::integral_constant<int, 1> one;
        if (vocab <= 8) return go(std::integral_constant<int, 8>{}, one);
        if (vocab <= 16) return go(std::integral_constant<int, 16>{}, one);
        if (vocab <= 32) return go(std::integral_constant<int, 32>{}, one);
        if (vocab <= 64) return go(std::integral_constant<int, 64>{}, one);
        return go(std::integral_constant<int, 64>{}, std::integral_constant<int, 4>{});
    });
}

}  // extern "C"
