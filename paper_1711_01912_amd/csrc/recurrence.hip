// Gated linear recurrence over rows of `width` channels, cut into sequences:
//
//   a = sigmoid(f + bias), z = 1 - a = sigmoid(-(f + bias)),  h_t = a_t h_{t-1} + z_t x_t
//
// z is formed directly, as 1 / (1 + e^(f + bias)), so that channels with a near 1 (long time scales) lose nothing.  A run of
// rows turns the state h that enters it into A h + H, with A the product of its a and H the state it ends in from zero: runs
// are taken side by side and joined.  Backward, with u_t = a_t g_t what flows into h_{t-1}:
//
//   g_t = dh_t + u_{t+1},  dx_t = z_t g_t,  df_t = g_t (h_{t-1} - x_t) a_t z_t,  u_t = a_t g_t
//
// the same kind of recurrence from the last row to the first; h_{t-1} is computed again from states kept by the forward pass.
// Rows are counted in the direction of the scan throughout ("position"): of a reversed scan, position 0 is the last row.
// States, products and sums are floats; a row's result is rounded once, to the element type.
//
// Bound by memory, and laid out to read every input once: a workgroup takes a tile of rows x 128 bytes of channels (a cache
// line of each row) into registers, 16 lanes a row, `kRun` rows a lane.  It publishes what its tile does to a state, looks
// back over the tiles before it until it meets a state that is known, publishes its own, and writes its rows.  Narrow and
// long tiles keep what is read in looking back small beside a tile's own bytes, and the number of tiles that the chain of
// states has to pass.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "policy.hpp"

namespace cpeval {

namespace {

constexpr int kLanes = 16;                          // lanes of a row: with 8 bytes each, 128 bytes
constexpr int kSides = kWave / kLanes;              // runs side by side in a wavefront
constexpr int kWaves = 8;
constexpr int kRuns = kWaves * kSides;              // runs of a workgroup, one behind the other
constexpr int kForwardRun = 16, kBackwardRun = 8;   // rows of a run, held in registers
template <typename T>
constexpr int kWide = 8 / sizeof(T);                // channels of a lane

// Where sequences begin, in positions
struct Sequences {
    const int32_t *ptr;      // [count + 1], or null: `count` equal parts of `each` rows
    int64_t rows, each;
    int32_t count;
    bool reverse;

    __device__ __forceinline__ int64_t start(int32_t j) const {
        if (!ptr) return each * j;
        return reverse ? rows - ptr[count - j] : (int64_t)ptr[j];
    }
    __device__ __forceinline__ int32_t number(int32_t j) const { return reverse ? count - 1 - j : j; }
    __device__ __forceinline__ int64_t row(int64_t position) const { return reverse ? rows - 1 - position : position; }

    // how many sequences start at or before `position`, by a whole wavefront: 64 probes a round.  Bounded, and within the
    // array, whatever it holds
    __device__ int32_t begun(int64_t position) const {
        if (!ptr) return each ? min(count, (int32_t)((uint32_t)position / (uint32_t)each) + 1) : count;
        const int lane = threadIdx.x & (kWave - 1);
        int32_t lo = 0, len = count;
        while (len > kWave) {
            const int32_t step = (len + kWave - 1) / kWave;
            const int64_t at = (int64_t)(lane + 1) * step - 1;
            const bool le = at < len && start(lo + (int32_t)at) <= position;
            const int32_t past = min(__popcll(__ballot(le)) * step, len);
            lo += past;
            len = min(step, len - past);
        }
        const bool le = lane < len && start(lo + lane) <= position;
        return lo + __popcll(__ballot(le));
    }
};

// The sequence starts among a wavefront's rows, of which each lane has the `run` from its own position on
template <int RUN>
struct Starts {
    static constexpr int kSpan = kSides * RUN;
    static_assert(kSpan <= 64, "a wavefront's rows are bits of a word");
    uint32_t first;          // bit i: the lane's i-th row is a sequence's first, or lies behind the last row; i = 0 .. RUN
    bool any;                // whether any lane of the wavefront has one, or less than RUN rows
    int32_t *begins, *ends;  // of the lane's rows: the sequence that begins with a marked row, the one that ends in front of it

    __device__ __forceinline__ void find(const Sequences &s, int64_t wave0, int wave, int side) {
        __shared__ int32_t lds[2][kWaves][kSpan + 1];
        const int lane = threadIdx.x & (kWave - 1);
        int32_t *first_of = lds[0][wave], *last_of = lds[1][wave];
        uint64_t bits = 0;
        bool next = false;               // of the row behind the wavefront's
        const int32_t lo = wave0 > 0 ? s.begun(wave0 - 1) : 0;
        bool some = false;
        for (int32_t j = lo; j < s.count; j += kWave) {
            const int64_t p = j + lane < s.count ? s.start(j + lane) : INT64_MAX;
            const bool in = p >= wave0 && p <= wave0 + kSpan && p <= s.rows;
            if (__ballot(in)) {
                if (!some) {
                    for (int q = lane; q <= kSpan; q += kWave) first_of[q] = INT32_MIN, last_of[q] = INT32_MAX;
                    some = true;
                }
                // (of sequences that begin at the same row, all but the last are empty)
                if (in) {
                    atomicMax(&first_of[p - wave0], j + lane);
                    atomicMin(&last_of[p - wave0], j + lane);
                }
                uint64_t mine = in && p < wave0 + kSpan ? 1ull << (p - wave0) : 0;
#pragma unroll
                for (int off = 1; off < kWave; off <<= 1) mine |= __shfl_xor((unsigned long long)mine, off);
                bits |= mine;
                next = next || __ballot(in && p == wave0 + kSpan);
            }
            if (__ballot(p > wave0 + kSpan)) break;
        }
        if (s.rows >= wave0 && s.rows <= wave0 + kSpan) {        // the row behind the last
            if (!some) {
                for (int q = lane; q <= kSpan; q += kWave) first_of[q] = INT32_MIN, last_of[q] = INT32_MAX;
                some = true;
            }
            if (lane == 0) atomicMin(&last_of[s.rows - wave0], s.count);
            if (s.rows < wave0 + kSpan) bits |= 1ull << (s.rows - wave0);
            else next = true;
        }
        any = some || s.rows < wave0 + kSpan;            // (also of wavefronts that lie behind the last row)
        first = (uint32_t)(bits >> (side * RUN)) & ((1u << RUN) - 1);
        const bool behind = side + 1 < kSides ? bits >> ((side + 1) * RUN) & 1 : next;
        first |= behind ? 1u << RUN : 0u;
        begins = first_of + side * RUN;
        ends = last_of + side * RUN;
    }
    // (in range whatever the pointers hold)
    __device__ __forceinline__ int64_t begun_by(const Sequences &s, int i) const { return s.number(min(max(begins[i], 0), s.count - 1)); }
    __device__ __forceinline__ int64_t ended_by(const Sequences &s, int i) const { return s.number(min(max(ends[i + 1] - 1, 0), s.count - 1)); }
};

// A sequence pointer that does not rise from 0 to `rows`: told in *status, by one workgroup.  (The scan itself stays inside
// its arrays whatever the pointers hold.)
__device__ void check_sequences(const Sequences &seq, int32_t *status) {
    __shared__ int bad;
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    if (seq.ptr) {
        for (int32_t j = threadIdx.x; j < seq.count; j += blockDim.x)
            if (seq.ptr[j] > seq.ptr[j + 1]) bad = 1;
        if (threadIdx.x == 0 && (seq.ptr[0] != 0 || seq.ptr[seq.count] != seq.rows)) bad = 1;
    }
    __syncthreads();
    if (threadIdx.x == 0) *status = bad ? CP_STATUS_BAD_SEQUENCE : CP_STATUS_OK;
}

// What rows do to the state that enters them: h -> A h + H, or h -> H whatever h where a sequence begins inside (A < 0).
// (Never 0 * h for that: what a sequence holds, a NaN included, stays in it.)
struct Effect {
    float A, H;
    __device__ __forceinline__ float of(float h) const { return A < 0 ? H : fmaf(A, h, H); }
};

__device__ __forceinline__ Effect then(Effect p, Effect q) {
    return q.A < 0 ? q : Effect{p.A < 0 ? p.A : p.A * q.A, fmaf(q.A, p.H, q.H)};
}

// An effect in memory that other workgroups wait for: one word, all ones until it is there.  A is never a NaN (where z is
// one, H is too), so no effect looks like that; and since a word is written whole, it needs no order with other memory.
constexpr uint64_t kNotYet = ~0ull;
__device__ __forceinline__ void publish(uint64_t *at, Effect e) {
    const uint64_t w = (uint64_t)__float_as_uint(e.H) << 32 | __float_as_uint(e.A);
    __hip_atomic_store(at, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t look(const uint64_t *at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ Effect effect_of(uint64_t w) { return {__uint_as_float((uint32_t)w), __uint_as_float((uint32_t)(w >> 32))}; }

__device__ __forceinline__ float keep_not(float f, float bias) { return fast_rcp(1.0f + fast_exp(f + bias)); }   // z

// (1 - z) h + z x, with h - z h rounded once: 1 - z, rounded, would be off by more than z where z is small
__device__ __forceinline__ float next(float z, float h, float x) { return fmaf(z, x, fmaf(-z, h, h)); }

// rows of [..][width] floats
template <int V>
__device__ __forceinline__ void start_from(float (&to)[V], const float *rows, int64_t row, int32_t width, int32_t c) {
#pragma unroll
    for (int k = 0; k < V; k++) to[k] = rows ? rows[row * width + c + k] : 0.0f;
}
template <int V>
__device__ __forceinline__ void put(float *rows, int64_t row, int32_t width, int32_t c, const float (&from)[V]) {
#pragma unroll
    for (int k = 0; k < V; k++) rows[row * width + c + k] = from[k];
}

// f for wavefronts with a sequence's start or the last row among their rows, or the same without looking for them
template <typename F>
__device__ __forceinline__ void either(bool any, F f) {
    if (any) f(std::true_type{});
    else f(std::false_type{});
}

// The compiler does not move instructions over this: left to itself it starts the exponentials of all rows at once and
// spills what they give.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

struct Scan {
    Sequences seq;
    int32_t width, strips, lookers;      // lookers: wavefronts that look back, kSides tiles each at a time
    int64_t tiles;
    const void *f, *x;
    int64_t ldf, ldx;
    const float *bias, *h0;
    uint32_t *ticket;                    // the next tile to be taken; null: one tile a strip
    uint64_t *words;                     // [tiles][strips][kLanes * V] effects
};

// A lane's place: its channels and its run.  The last lane of a row that is no multiple of V takes its last V channels, some
// of them as its neighbour does, to the same values.
template <typename T, int V>
struct Place {
    int64_t tile, wave0, p0;
    int32_t strip, c;
    int lane, side, wave, run;
    bool live;

    template <int RUN>
    __device__ __forceinline__ void take(const Scan &s, bool backward) {
        __shared__ uint32_t ticket;
        lane = threadIdx.x & (kLanes - 1);
        side = threadIdx.x / kLanes & (kSides - 1);
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        run = wave * kSides + side;
        uint32_t n = blockIdx.x;
        if (s.ticket) {
            // in the order in which workgroups come to life: one waits for none but those that live already
            if (threadIdx.x == 0) ticket = atomicAdd(s.ticket, 1u);
            __syncthreads();
            n = __builtin_amdgcn_readfirstlane(ticket);
        }
        tile = n / (uint32_t)s.strips;
        strip = (int32_t)(n - (uint32_t)tile * (uint32_t)s.strips);
        if (backward) tile = s.tiles - 1 - tile;
        wave0 = tile * (kRuns * RUN) + wave * (kSides * RUN);
        p0 = wave0 + side * RUN;
        c = (strip * kLanes + lane) * V;
        live = c < s.width;
        c = live ? min(c, s.width - V) : 0;
    }
    __device__ __forceinline__ uint64_t *word(const Scan &s, int64_t of) const { return s.words + ((of * s.strips + strip) * kLanes + lane) * V; }
};

// V values as the words they are loaded in.  (As values of 16 bits the compiler gives each a register of its own.)
template <typename T, int V>
struct Raw {
    uint32_t w[(V * sizeof(T) + 3) / 4];

    __device__ __forceinline__ void load(const T *p) {
        const Pack<T, V> v = load_pack<T, V>(p);
        w[0] = 0;
        __builtin_memcpy(w, &v, sizeof(v));
    }
    __device__ __forceinline__ float operator[](int k) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[k]);
        else if constexpr (std::is_same_v<T, bf16>) return __uint_as_float(k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
        else return (float)__builtin_bit_cast(f16, (uint16_t)(k & 1 ? w[k / 2] >> 16 : w[k / 2]));
    }
    __device__ __forceinline__ void fill(uint32_t word) {
#pragma unroll
        for (uint32_t &one : w) one = word;
    }
    // what was computed from them (conversions, z) is computed again where it is needed again: the compiler takes them as
    // unknown from here on.  Kept in registers it would be twice the values themselves, and half the wavefronts.
    __device__ __forceinline__ void forget() {
#pragma unroll
        for (uint32_t &one : w) asm volatile("" : "+v"(one));
    }
};
template <typename T>
constexpr uint32_t kInfinite = sizeof(T) == 4 ? 0x7f800000u : std::is_same_v<T, bf16> ? 0x7f807f80u : 0x7c007c00u;

// A lane's run of a matrix's rows: what all lanes of the wavefront share of an address is kept in scalar registers, and a
// lane's own part in one.
template <typename T, int V, int RUN>
struct Run {
    const char *base;        // the lowest row that a lane of the wavefront has at its i = 0, column 0
    int64_t step;            // bytes from a lane's row to its next one
    uint32_t off;

    __device__ __forceinline__ Run(const void *at, int64_t ld, const Sequences &seq, const Place<T, V> &p) {
        const int side = seq.reverse ? kSides - 1 - p.side : p.side;
        base = (const char *)((const T *)at + (seq.reverse ? seq.rows - 1 - p.wave0 - (kSides - 1) * RUN : p.wave0) * ld);
        step = (seq.reverse ? -ld : ld) * (int64_t)sizeof(T);
        off = (uint32_t)((side * RUN * (uint32_t)ld + p.c) * sizeof(T));
    }
    __device__ __forceinline__ T *row(int i) const { return (T *)(base + i * step + off); }

    // rows behind the last are `word` throughout
    __device__ __forceinline__ void load(Raw<T, V> (&to)[RUN], bool full, int rows, uint32_t word) const {
        if (full) {
#pragma unroll
            for (int i = 0; i < RUN; i++) to[i].load(row(i));
        } else {
#pragma unroll
            for (int i = 0; i < RUN; i++) {
                to[i].fill(word);
                if (i < rows) to[i].load(row(i));
            }
        }
    }
};

template <typename T, int V, int RUN>
__device__ __forceinline__ void forget(Raw<T, V> (&of)[RUN]) {
#pragma unroll
    for (int i = 0; i < RUN; i++) of[i].forget();
}

// From the effects of a workgroup's runs (forward: in their order, backward: in the opposite one) to the state that enters
// each: they are joined inside the wavefronts, then over the tiles before, and applied from there.  What has to wait
// meanwhile waits in LDS: registers are full of rows.
template <typename T, int V, bool BACK>
struct Join {
    Effect (*waves)[V][kLanes];          // what each wavefront's runs do, in the order of the chain
    Effect (*before)[kWaves * kWave];    // what the runs of the wavefront before the lane's do

    static __device__ __forceinline__ int order(int i, int of) { return BACK ? of - 1 - i : i; }

    __device__ __forceinline__ void inside(const Place<T, V> &p, const Effect (&e)[V]) {
        __shared__ Effect lds_waves[kWaves][V][kLanes], lds_before[V][kWaves * kWave];
        waves = lds_waves;
        before = lds_before;
        const int side = order(p.side, kSides), here = threadIdx.x & (kWave - 1);
#pragma unroll
        for (int k = 0; k < V; k++) {
            Effect sum = e[k];
#pragma unroll
            for (int d = 1; d < kSides; d <<= 1) {
                const int from = here + (BACK ? d : -d) * kLanes;
                const Effect o = {__shfl(sum.A, from), __shfl(sum.H, from)};
                sum = side >= d ? then(o, sum) : sum;
            }
            if (side == kSides - 1) waves[order(p.wave, kWaves)][k][p.lane] = sum;
            const int from = here + (BACK ? kLanes : -kLanes);
            const Effect o = {__shfl(sum.A, from), __shfl(sum.H, from)};
            before[k][threadIdx.x] = side ? o : Effect{1.0f, 0.0f};
        }
        __syncthreads();
    }

    // what the whole tile does to a channel
    __device__ __forceinline__ Effect whole(const Place<T, V> &p, int k) const {
        Effect all = waves[0][k][p.lane];
        for (int w = 1; w < kWaves; w++) all = then(all, waves[w][k][p.lane]);
        return all;
    }

    // the state that enters the tile
    __device__ __forceinline__ void behind(const Place<T, V> &p, const Scan &s, float (&state)[V]) {
        __shared__ Effect lds[kRuns][V][kLanes];
        const int64_t tile = BACK ? s.tiles - 1 - p.tile : p.tile;          // in the order of the chain
        const bool tells = p.run == 0 && p.live && tile + 1 < s.tiles;
        if (tells) {
#pragma unroll
            for (int k = 0; k < V; k++) {
                const Effect all = whole(p, k);
                publish(p.word(s, p.tile) + k, {tile ? all.A : -1.0f, all.H});
            }
        }
        Effect all[V];
#pragma unroll
        for (int k = 0; k < V; k++) all[k] = {1.0f, 0.0f};
        const int at_once = s.lookers * kSides;
        for (int64_t near = tile - 1; near >= 0; near -= at_once) {
            if (p.wave < s.lookers) {
                const int64_t of = near - p.run;
                const bool there = of >= 0 && p.live;
                const uint64_t *at = p.word(s, there ? BACK ? s.tiles - 1 - of : of : p.tile);
#pragma unroll
                for (int k = 0; k < V; k++) {
                    uint64_t w = there ? look(at + k) : 0;
                    while (w == kNotYet) w = look(at + k);
                    lds[p.run][k][p.lane] = there ? effect_of(w) : Effect{-1.0f, 0.0f};
                }
            }
            __syncthreads();
            bool known = false;
            for (int q = 0; q < at_once && !known; q++) {
                known = true;
#pragma unroll
                for (int k = 0; k < V; k++) {
                    all[k] = then(lds[q][k][p.lane], all[k]);
                    known &= all[k].A < 0;
                }
                known = __all(known);
            }
            if (known) break;            // (every wavefront sees the same)
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < V; k++) state[k] = tile ? all[k].H : 0.0f;
        if (tells && tile) {
#pragma unroll
            for (int k = 0; k < V; k++) publish(p.word(s, p.tile) + k, {-1.0f, whole(p, k).of(state[k])});
        }
    }

    // from the state that enters the tile to the one that enters the lane's run
    __device__ __forceinline__ void enter(const Place<T, V> &p, float (&state)[V]) const {
        const int wave = order(p.wave, kWaves);
        for (int w = 0; w < wave; w++) {
#pragma unroll
            for (int k = 0; k < V; k++) state[k] = waves[w][k][p.lane].of(state[k]);
        }
#pragma unroll
        for (int k = 0; k < V; k++) state[k] = before[k][threadIdx.x].of(state[k]);
    }
};

template <typename T, int V>
__global__ __launch_bounds__(kWaves *kWave, 4) void scan_kernel(Scan s, T *h, int64_t ldh, float *last, float *carry, int32_t *status) {
    constexpr int RUN = kForwardRun;
    Place<T, V> p;
    p.template take<RUN>(s, false);
    const Sequences &seq = s.seq;
    const int32_t c = p.c;
    const bool full = p.wave0 + kSides * RUN <= seq.rows;
    const int64_t left = seq.rows - p.p0;
    const int rows = left <= 0 ? 0 : left < RUN ? (int)left : RUN;

    Raw<T, V> fr[RUN], xr[RUN];
    // (z is 0 where f is infinite: rows behind the last leave the state as it is)
    Run<T, V, RUN>(s.f, s.ldf, seq, p).load(fr, full, rows, kInfinite<T>);
    Run<T, V, RUN>(s.x, s.ldx, seq, p).load(xr, full, rows, 0u);
    Starts<RUN> starts;
    starts.find(seq, p.wave0, p.wave, p.side);
    if (status && blockIdx.x == 0) check_sequences(seq, status);
    float bias[V];
#pragma unroll
    for (int k = 0; k < V; k++) bias[k] = s.bias ? s.bias[c + k] : 0.0f;

    const uint32_t mine = (1u << rows) - 1;
    const bool begins = starts.first & mine;
    float state[V], A[V];
#pragma unroll
    for (int k = 0; k < V; k++) state[k] = 0.0f, A[k] = 1.0f;
    either(starts.any, [&](auto any) {
#pragma unroll
        for (int i = 0; i < RUN; i++) {
            if (any && (starts.first & mine) >> i & 1) start_from<V>(state, s.h0, s.h0 ? starts.begun_by(seq, i) : 0, s.width, c);
#pragma unroll
            for (int k = 0; k < V; k++) {
                const float z = keep_not(fr[i][k], bias[k]);
                state[k] = next(z, state[k], xr[i][k]);
                A[k] = fmaf(-z, A[k], A[k]);
            }
            in_order();
        }
    });
    Effect e[V];
#pragma unroll
    for (int k = 0; k < V; k++) e[k] = {begins ? -1.0f : fmaxf(A[k], 0.0f), state[k]};
    forget<T, V, RUN>(fr);
    forget<T, V, RUN>(xr);
    Join<T, V, false> join;
    join.inside(p, e);
    if (s.ticket) join.behind(p, s, state);
    else
#pragma unroll
        for (int k = 0; k < V; k++) state[k] = 0.0f;
    join.enter(p, state);

    if (carry && p.live && p.p0 % CP_RECURRENCE_CHUNK == 0 && rows > 0) {
#pragma unroll
        for (int k = 0; k < V; k++) carry[p.p0 / CP_RECURRENCE_CHUNK * s.width + c + k] = state[k];
    }
    const Run<T, V, RUN> to(h, ldh, seq, p);
    either(starts.any, [&](auto any) {
#pragma unroll
        for (int i = 0; i < RUN; i++) {
            if (any && (starts.first & mine) >> i & 1) start_from<V>(state, s.h0, s.h0 ? starts.begun_by(seq, i) : 0, s.width, c);
            Pack<T, V> out;
#pragma unroll
            for (int k = 0; k < V; k++) {
                state[k] = next(keep_not(fr[i][k], bias[k]), state[k], xr[i][k]);
                out.v[k] = (T)state[k];
            }
            in_order();
            if (!any) {          // (and then all rows are there)
                if (p.live) store_pack<T, V>(to.row(i), out);
            } else if (p.live && i < rows) {
                store_pack<T, V>(to.row(i), out);
                if (last && (starts.first >> (i + 1) & 1)) put<V>(last, starts.ended_by(seq, i), s.width, c, state);
            }
        }
    });
    // a sequence without rows ends in the state that it begins with
    if (last && p.live && (seq.ptr || seq.each == 0)) {
        for (int64_t j = p.tile * kRuns + p.run; j < seq.count; j += s.tiles * kRuns) {
            if (seq.ptr && seq.ptr[j] < seq.ptr[j + 1]) continue;
#pragma unroll
            for (int k = 0; k < V; k++) last[j * s.width + c + k] = s.h0 ? s.h0[j * s.width + c + k] : 0.0f;
        }
    }
}

template <typename T, int V>
__global__ __launch_bounds__(kWaves *kWave, 4) void scan_backward_kernel(Scan s, const T *dh, int64_t lddh, const float *dlast, const float *carry,
                                                                         T *df, int64_t lddf, T *dx, int64_t lddx, float *dbias_part,
                                                                         float *dh0, int32_t *status) {
    constexpr int RUN = kBackwardRun;
    static_assert(kRuns * RUN % CP_RECURRENCE_CHUNK == 0, "a tile begins where a state was kept");
    Place<T, V> p;
    p.template take<RUN>(s, true);
    const Sequences &seq = s.seq;
    const int32_t c = p.c;
    const bool full = p.wave0 + kSides * RUN <= seq.rows;
    const int64_t left = seq.rows - p.p0;
    const int rows = left <= 0 ? 0 : left < RUN ? (int)left : RUN;

    Raw<T, V> fr[RUN], xr[RUN], dr[RUN];
    Run<T, V, RUN>(s.f, s.ldf, seq, p).load(fr, full, rows, kInfinite<T>);
    Run<T, V, RUN>(dh, lddh, seq, p).load(dr, full, rows, 0u);
    Run<T, V, RUN>(s.x, s.ldx, seq, p).load(xr, full, rows, 0u);
    float state[V], bias[V];
#pragma unroll
    for (int k = 0; k < V; k++) {
        bias[k] = s.bias ? s.bias[c + k] : 0.0f;
        // the state that enters the tile was kept
        state[k] = p.tile ? carry[p.tile * (kRuns * RUN / CP_RECURRENCE_CHUNK) * s.width + c + k] : 0.0f;
    }
    Starts<RUN> starts;
    starts.find(seq, p.wave0, p.wave, p.side);
    if (status && blockIdx.x == 0) check_sequences(seq, status);

    const uint32_t mine = (1u << rows) - 1, firsts = starts.first & mine, lasts = starts.first >> 1 & mine;
    float u[V];
    Effect e[V], d[V];
    {
        float z[RUN][V], run[V], A[V];
#pragma unroll
        for (int k = 0; k < V; k++) run[k] = 0.0f, A[k] = 1.0f, u[k] = 0.0f;
        either(starts.any, [&](auto any) {
#pragma unroll
            for (int i = 0; i < RUN; i++) {
                if (any && firsts >> i & 1) start_from<V>(run, s.h0, s.h0 ? starts.begun_by(seq, i) : 0, s.width, c);
#pragma unroll
                for (int k = 0; k < V; k++) {
                    z[i][k] = keep_not(fr[i][k], bias[k]);
                    run[k] = next(z[i][k], run[k], xr[i][k]);
                    A[k] = fmaf(-z[i][k], A[k], A[k]);
                }
                in_order();
            }
#pragma unroll
            for (int i = RUN - 1; i >= 0; i--) {
                if (any && lasts >> i & 1) start_from<V>(u, dlast, dlast ? starts.ended_by(seq, i) : 0, s.width, c);
#pragma unroll
                for (int k = 0; k < V; k++) {
                    const float g = u[k] + dr[i][k];
                    u[k] = fmaf(-z[i][k], g, g);
                }
            }
        });
#pragma unroll
        for (int k = 0; k < V; k++) {
            const float a = fmaxf(A[k], 0.0f);
            e[k] = {firsts ? -1.0f : a, run[k]};
            d[k] = {lasts ? -1.0f : a, u[k]};
        }
    }
    forget<T, V, RUN>(fr);
    forget<T, V, RUN>(xr);
    forget<T, V, RUN>(dr);
    {
        Join<T, V, true> join;
        join.inside(p, d);
        if (s.ticket) join.behind(p, s, u);
        else
#pragma unroll
            for (int k = 0; k < V; k++) u[k] = 0.0f;
        join.enter(p, u);
    }
    {
        Join<T, V, false> join;
        join.inside(p, e);
        join.enter(p, state);
    }
    float before[RUN][V], sum[V];
#pragma unroll
    for (int k = 0; k < V; k++) sum[k] = 0.0f;
    const Run<T, V, RUN> to_f(df, lddf, seq, p), to_x(dx, lddx, seq, p);
    either(starts.any, [&](auto any) {
#pragma unroll
        for (int i = 0; i < RUN; i++) {
            if (any && firsts >> i & 1) start_from<V>(state, s.h0, s.h0 ? starts.begun_by(seq, i) : 0, s.width, c);
#pragma unroll
            for (int k = 0; k < V; k++) {
                before[i][k] = state[k];
                state[k] = next(keep_not(fr[i][k], bias[k]), state[k], xr[i][k]);
            }
            in_order();
        }
        forget<T, V, RUN>(fr);
        forget<T, V, RUN>(xr);
#pragma unroll
        for (int i = RUN - 1; i >= 0; i--) {
            if (any && lasts >> i & 1) start_from<V>(u, dlast, dlast ? starts.ended_by(seq, i) : 0, s.width, c);
            Pack<T, V> of, ox;
#pragma unroll
            for (int k = 0; k < V; k++) {
                const float ef = fast_exp(fr[i][k] + bias[k]), z = fast_rcp(1.0f + ef);
                const float a = ef < 1.0f ? ef * z : 1.0f - z;      // (exact to its size at both ends)
                const float g = dr[i][k] + u[k], gz = g * z;
                const float v = gz * a * (before[i][k] - xr[i][k]);
                ox.v[k] = (T)gz;
                of.v[k] = (T)v;
                sum[k] += !any || i < rows ? v : 0.0f;
                u[k] = g - gz;
            }
            in_order();
            if (p.live && (!any || i < rows)) {
                store_pack<T, V>(to_x.row(i), ox);
                store_pack<T, V>(to_f.row(i), of);
                if (any && dh0 && firsts >> i & 1) put<V>(dh0, starts.begun_by(seq, i), s.width, c, u);
            }
        }
    });
    if (dbias_part) {
        __shared__ float lds[kWaves][V][kLanes];
#pragma unroll
        for (int k = 0; k < V; k++) {
            sum[k] += __shfl_xor(sum[k], kLanes);
            sum[k] += __shfl_xor(sum[k], 2 * kLanes);
            if (p.side == 0) lds[p.wave][k][p.lane] = sum[k];
        }
        __syncthreads();
        if (p.run == 0 && p.live) {
#pragma unroll
            for (int k = 0; k < V; k++) {
                float all = 0.0f;
                for (int w = 0; w < kWaves; w++) all += lds[w][k][p.lane];
                dbias_part[p.tile * s.width + c + k] = all;
            }
        }
    }
    if (dh0 && p.live && (seq.ptr || seq.each == 0)) {
        for (int64_t j = p.tile * kRuns + p.run; j < seq.count; j += s.tiles * kRuns) {
            if (seq.ptr && seq.ptr[j] < seq.ptr[j + 1]) continue;
#pragma unroll
            for (int k = 0; k < V; k++) dh0[j * s.width + c + k] = dlast ? dlast[j * s.width + c + k] : 0.0f;
        }
    }
}

// No effect is there yet, and no tile taken.
__global__ __launch_bounds__(256) void clear_words_kernel(uint32_t *ticket, uint64_t *words, int64_t count) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) words[i] = kNotYet;
}

// sums over rows of the tiles' sums, 16 columns a workgroup, in a fixed order and in 64 bits
__global__ __launch_bounds__(1024) void column_sum_kernel(const float *part, int64_t rows, int32_t width, float *out) {
    __shared__ double lds[64][16];
    const int lane = threadIdx.x & 15, row = threadIdx.x / 16;
    const int32_t c = blockIdx.x * 16 + lane;
    double sum = 0.0;
    if (c < width) {
#pragma unroll 4
        for (int64_t i = row; i < rows; i += 64) sum += part[i * width + c];
    }
    lds[row][lane] = sum;
    __syncthreads();
    if (row == 0 && c < width) {
        for (int w = 1; w < 64; w++) sum += lds[w][lane];
        out[c] = (float)sum;
    }
}

template <typename T, int V>
__global__ __launch_bounds__(256) void step_kernel(int32_t count, int32_t width, const T *f, int64_t ldf, const T *x, int64_t ldx,
                                                   const float *bias, float *state, int32_t num_slots, const int32_t *slots, T *h,
                                                   int64_t ldh, int32_t *status) {
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V;
    for (int64_t s = blockIdx.y; s < count; s += gridDim.y) {
        const int32_t slot = slots ? slots[s] : (int32_t)s;
        const bool bad = slot >= num_slots;
        if (bad && status && threadIdx.x == 0 && blockIdx.x == 0) atomicOr(status, CP_STATUS_BAD_SLOT);
        if (c >= width) continue;
        Pack<T, V> out;
        if (slot < 0 || bad) {
#pragma unroll
            for (int k = 0; k < V; k++) out.v[k] = (T)0.0f;
        } else {
            const Pack<T, V> fv = load_pack<T, V>(f + s * ldf + c), xv = load_pack<T, V>(x + s * ldx + c);
            float *at = state + (int64_t)slot * width + c;
            Pack<float, V> st = load_pack<float, V>(at);
#pragma unroll
            for (int k = 0; k < V; k++) {
                const float z = keep_not((float)fv.v[k], bias ? bias[c + k] : 0.0f);
                st.v[k] = next(z, st.v[k], (float)xv.v[k]);
                out.v[k] = (T)st.v[k];
            }
            store_pack<float, V>(at, st);
        }
        store_pack<T, V>(h + s * ldh + c, out);
    }
}

__global__ void set_status_kernel(int32_t *status, int32_t value) { *status = value; }

// rows apart by at least their width, and so little that a wavefront's rows lie within 32 bits of bytes
bool distances(int32_t width, std::initializer_list<int64_t> ld) {
    for (int64_t d : ld)
        if (d < width || d > CP_RECURRENCE_MAX_DISTANCE) return false;
    return true;
}

int check_scan(int64_t rows, int32_t width, int32_t num_seq, const int32_t *seq_ptr, int type, int reverse) {
    if (!known_type(type) || (reverse != 0 && reverse != 1)) return CP_ERR_ARG;
    if (rows < 0 || rows > INT32_MAX || width < 1 || width > CP_RECURRENCE_MAX_WIDTH || num_seq < 1) return CP_ERR_SIZE;
    if (!seq_ptr && rows % num_seq) return CP_ERR_SIZE;
    return CP_OK;
}

int64_t tiles_of(int64_t rows, int run) { return std::max<int64_t>(1, (rows + kRuns * run - 1) / (kRuns * run)); }

// A ticket, and an effect for each tile and channel, channels counted up to whole strips of the widest type's lanes
size_t words_bytes(int64_t rows, int32_t width, bool backward) {
    const size_t channels = ((size_t)width + kLanes * kWide<bf16> - 1) / (kLanes * kWide<bf16>) * (kLanes * kWide<bf16>);
    return kPolicyAlign + align_up(tiles_of(rows, backward ? kBackwardRun : kForwardRun) * channels * sizeof(uint64_t));
}
size_t part_bytes(int64_t rows, int32_t width) { return align_up((size_t)tiles_of(rows, kBackwardRun) * width * sizeof(float)); }

// Wavefronts that look back.  The chain of states passes as many tiles a round as are looked at; the fewer strips there are,
// the more tiles of each are under way at once, and the faster it has to be.
int lookers_of(int32_t strips) { return std::max(1, std::min(kWaves, 32 / strips)); }

void split_over(Scan &s, int run, int v, void *workspace) {
    s.strips = (s.width + kLanes * v - 1) / (kLanes * v);
    s.tiles = tiles_of(s.seq.rows, run);
    s.lookers = lookers_of(s.strips);
    s.ticket = s.tiles > 1 ? (uint32_t *)workspace : nullptr;
    s.words = s.tiles > 1 ? (uint64_t *)((char *)workspace + kPolicyAlign) : nullptr;
}

void clear_words(const Scan &s, int v, hipStream_t stream) {
    const int64_t count = s.tiles * s.strips * kLanes * v;
    hipLaunchKernelGGL(clear_words_kernel, dim3((unsigned)std::min<int64_t>((count + 255) / 256, 2048)), dim3(256), 0, stream, s.ticket, s.words, count);
}

}  // namespace

}  // namespace cpeval

using namespace cpeval;

extern "C" {

int cp_recurrence_workspace_bytes(int64_t rows, int32_t width, int backward, size_t *out_bytes) {
    if (!out_bytes) return CP_ERR_NULL;
    if (rows < 0 || rows > INT32_MAX || width < 1 || width > CP_RECURRENCE_MAX_WIDTH) return CP_ERR_SIZE;
    *out_bytes = words_bytes(rows, width, backward != 0) + (backward ? part_bytes(rows, width) : 0);
    return CP_OK;
}

int cp_recurrence(int64_t rows, int32_t width, int32_t num_seq, const int32_t *seq_ptr, int type, int reverse, const void *f,
                  int64_t ldf, const void *x, int64_t ldx, const float *bias, const float *h0, void *h, int64_t ldh, float *last,
                  float *carry, void *workspace, size_t workspace_bytes, void *stream, int32_t *status_out) {
    int rc = check_scan(rows, width, num_seq, seq_ptr, type, reverse);
    if (rc) return rc;
    if ((rows > 0 && (!f || !x || !h)) || (seq_ptr && !status_out)) return CP_ERR_NULL;
    if (rows > 1 && !distances(width, {ldf, ldx, ldh})) return CP_ERR_SIZE;
    if (rows > CP_RECURRENCE_CHUNK) {
        if (!workspace) return CP_ERR_NULL;
        if ((uintptr_t)workspace % kPolicyAlign || workspace_bytes < words_bytes(rows, width, false)) return CP_ERR_WORKSPACE;
    }
    Scan s{};
    s.seq = {seq_ptr, rows, rows / num_seq, num_seq, reverse != 0};
    s.width = width;
    s.f = f, s.ldf = ldf, s.x = x, s.ldx = ldx, s.bias = bias, s.h0 = h0;
    const hipStream_t st = (hipStream_t)stream;
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        auto go = [&](auto v) {
            constexpr int V = decltype(v)::value;
            split_over(s, kForwardRun, V, workspace);
            if (s.tiles * s.strips > INT32_MAX) return (int)CP_ERR_SIZE;
            if (s.ticket) clear_words(s, V, st);
            hipLaunchKernelGGL((scan_kernel<T, V>), dim3((unsigned)(s.tiles * s.strips)), dim3(kWaves * kWave), 0, st, s, (T *)h, ldh, last, carry,
                               seq_ptr ? status_out : nullptr);
            return launched();
        };
        if (width >= kWide<T>) return go(std::integral_constant<int, kWide<T>>{});
        return go(std::integral_constant<int, 1>{});
    });
}

int cp_recurrence_backward(int64_t rows, int32_t width, int32_t num_seq, const int32_t *seq_ptr, int type, int reverse,
                           const void *dh, int64_t lddh, const float *dlast, const void *f, int64_t ldf, const void *x, int64_t ldx,
                           const float *bias, const float *h0, const float *carry, void *df, int64_t lddf, void *dx, int64_t lddx,
                           float *dbias, float *dh0, void *workspace, size_t workspace_bytes, void *stream, int32_t *status_out) {
    int rc = check_scan(rows, width, num_seq, seq_ptr, type, reverse);
    if (rc) return rc;
    if ((rows > 0 && (!dh || !f || !x || !df || !dx)) || (seq_ptr && !status_out)) return CP_ERR_NULL;
    if (rows > 1 && !distances(width, {lddh, ldf, ldx, lddf, lddx})) return CP_ERR_SIZE;
    const bool split = rows > CP_RECURRENCE_CHUNK;
    if (split && !carry) return CP_ERR_NULL;
    if (split || dbias) {
        if (!workspace) return CP_ERR_NULL;
        if ((uintptr_t)workspace % kPolicyAlign || workspace_bytes < words_bytes(rows, width, true) + part_bytes(rows, width)) return CP_ERR_WORKSPACE;
    }
    float *part = dbias ? (float *)((char *)workspace + words_bytes(rows, width, true)) : nullptr;
    Scan s{};
    s.seq = {seq_ptr, rows, rows / num_seq, num_seq, reverse != 0};
    s.width = width;
    s.f = f, s.ldf = ldf, s.x = x, s.ldx = ldx, s.bias = bias, s.h0 = h0;
    const hipStream_t st = (hipStream_t)stream;
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        auto go = [&](auto v) {
            constexpr int V = decltype(v)::value;
            split_over(s, kBackwardRun, V, workspace);
            if (s.tiles * s.strips > INT32_MAX) return (int)CP_ERR_SIZE;
            if (s.ticket) clear_words(s, V, st);
            hipLaunchKernelGGL((scan_backward_kernel<T, V>), dim3((unsigned)(s.tiles * s.strips)), dim3(kWaves * kWave), 0, st, s, (const T *)dh, lddh,
                               dlast, carry, (T *)df, lddf, (T *)dx, lddx, part, dh0, seq_ptr ? status_out : nullptr);
            if (dbias)
                hipLaunchKernelGGL(column_sum_kernel, dim3((width + 15) / 16), dim3(1024), 0, st, part, s.tiles, width, dbias);
            return launched();
        };
        if (width >= kWide<T>) return go(std::integral_constant<int, kWide<T>>{});
        return go(std::integral_constant<int, 1>{});
    });
}

int cp_recurrence_step(int32_t num_seq, int32_t width, int type, const void *f, int64_t ldf, const void *x, int64_t ldx,
                       const float *bias, float *state, int32_t num_slots, const int32_t *slots, void *h, int64_t ldh, void *stream,
                       int32_t *status_out) {
    if (!known_type(type)) return CP_ERR_ARG;
    if (num_seq < 0 || num_slots < 1 || width < 1 || width > CP_RECURRENCE_MAX_WIDTH || (!slots && num_seq > num_slots)) return CP_ERR_SIZE;
    if ((num_seq > 0 && (!f || !x || !h)) || !state || (slots && !status_out)) return CP_ERR_NULL;
    if (num_seq > 1 && !distances(width, {ldf, ldx, ldh})) return CP_ERR_SIZE;
    const hipStream_t st = (hipStream_t)stream;
    if (slots) hipLaunchKernelGGL(set_status_kernel, dim3(1), dim3(1), 0, st, status_out, CP_STATUS_OK);
    if (num_seq == 0) return launched();
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        auto go = [&](auto v) {
            constexpr int V = decltype(v)::value;
            const dim3 grid((unsigned)((width + 256 * V - 1) / (256 * V)), (unsigned)std::min(num_seq, 65535));
            hipLaunchKernelGGL((step_kernel<T, V>), grid, dim3(256), 0, st, num_seq, width, (const T *)f, ldf, (const T *)x, ldx, bias, state,
                               num_slots, slots, (T *)h, ldh, status_out);
            return launched();
        };
        // (no two lanes may share a channel here: its state is read and written)
        if (width % 4 == 0) return go(std::integral_constant<int, 4>{});
        return go(std::integral_constant<int, 1>{});
    });
}

}  // extern "C"
