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
// the same kind of recurrence from the last row to the first; h_{t-1} is computed again from states kept by the forward pass:
// one per 128 rows, of which a tile's first, every second, is read.
// Rows are counted in the direction of the scan throughout ("position"): of a reversed scan, position 0 is the last row.
// States, products and sums are floats, and a result is rounded once, to the element type; dbias is summed in floats over a
// tile's 256 rows and in 64 bits over tiles, which leaves it off by less than its terms are.
//
// Bound by memory, and laid out to read every input once: a workgroup takes a tile of rows x 128 bytes of channels (a cache
// line of each row) into registers, two channels a lane.  It publishes what its tile does to a state, looks
// at what the tiles of its group before it do, waits for the state that enters the group, and writes its rows.  Narrow and
// long tiles keep what is read in looking back small beside a tile's own bytes, and the number of groups that the chain of
// states has to pass.  A million rows of 256 bf16 channels: 358 us forward and 605 backward, 4.2 TB/s both, where a copy reaches
// 5.1 (the forward kernel keeps 28 of its registers in scratch memory); 65536 x 1024 forward 103 us (3.9 TB/s), where a tile's wait
// for the state of its group shows, with two workgroups on a compute unit at 84 registers a lane.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "policy.hpp"

namespace cpeval {

namespace {

constexpr int kWaves = 8;
constexpr int kLooks = 2;                               // tiles that a lane looks at
constexpr int kWide = 2;                                // channels of a lane (of a width of one: one)
// Rows of a wavefront.  Forward, of 16-bit types, short spans need two thirds of the registers and long ones half the groups that
// the chain of states passes.  us a call with 32 and with 64 rows, bf16:
//   rows         65536      300000     400000     500000     700000     1000000
//   x 64       21 / 29    58 / 65    75 / 77    91 / 87   117 / 106    161 / 132
//   x 256      39 / 42   128 / 136  163 / 163  202 / 194  276 / 252    390 / 340
//   x 1024    100 / 121  402 / 378  533 / 486  661 / 596  920 / 817   1320 / 1157
// and 300000 x 75 fp16 76 and 90.  (At 1,024 channels the two meet below 300,000 rows: the line is 6 to 9 % off from there on.)
// Floats, of which a lane has half as many rows, take long ones: 65536 x 1024 149 us (short: 163), 500000 x 256 275 (329), a
// million x 64 161 (201), 300000 x 75 99 (107); 52710 x 333 74 (72) as one sequence, 65 (68) as 37.
constexpr int kShortSpan = 32, kLongSpan = 64, kBackwardSpan = 32;
constexpr int64_t kLongChain = 500000;                  // rows from which on spans are long
constexpr int forward_span(int64_t rows, size_t bytes) { return bytes == 2 && rows < kLongChain ? kShortSpan : kLongSpan; }

// How a wavefront's lanes share its rows: 128 bytes of each, kSides runs of them side by side, held in registers
template <typename T>
struct Shape {
    static constexpr int kLanes = 128 / (kWide * (int)sizeof(T)), kSides = kWave / kLanes, kRuns = kWaves * kSides;
    static constexpr int kBackwardRun = kBackwardSpan / kSides;
};

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

// Whether all of a tile's rows are there and lie inside one sequence, which neither begins nor ends with them
__device__ __forceinline__ bool is_inside(const Sequences &s, int64_t first, int64_t rows) {
    return first > 0 && first + rows < s.rows && s.begun(first - 1) == s.begun(first + rows);
}

// The sequence starts among a wavefront's rows, of which each lane has the `run` from its own position on
template <int RUN, int SIDES>
struct Starts {
    static constexpr int kSpan = SIDES * RUN;
    static_assert(kSpan <= 64, "a wavefront's rows are bits of a word");
    uint64_t first;          // bit i: the lane's i-th row is a sequence's first, or lies behind the last row; i = 0 .. RUN
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
            const int64_t p = lane < s.count - j ? s.start(j + lane) : INT64_MAX;
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
        first = bits >> (side * RUN) & ((1ull << RUN) - 1);
        const bool behind = side + 1 < SIDES ? bits >> (side + 1 < SIDES ? (side + 1) * RUN : 0) & 1 : next;
        first |= behind ? 1ull << RUN : 0ull;
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

// e^(f + bias), with the bias in units of ln 2, and z = 1 / (1 + e^(f + bias))
__device__ __forceinline__ float odds(float f, float bias2) { return __builtin_amdgcn_exp2f(fmaf(f, kLog2e, bias2)); }
__device__ __forceinline__ float keep_not(float f, float bias2) { return fast_rcp(1.0f + odds(f, bias2)); }

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

struct Scan {
    Sequences seq;
    int32_t width, strips, lookers;      // lookers: wavefronts that look back, kSides tiles each at a time
    int64_t tiles;
    const void *f, *x;
    int64_t ldf, ldx;
    const float *bias, *h0;
    uint32_t *ticket;                    // the next tile to be taken; null: one tile a strip
    uint64_t *words;                     // [tiles][strips][kLanes * V] effects, then as many for the states that enter groups
};

// A lane's place: its channels and its run.  The last lane of a row that is no multiple of V takes its last V channels, some
// of them as its neighbour does, to the same values.
template <typename T, int V>
struct Place : Shape<T> {
    using Shape<T>::kLanes;
    using Shape<T>::kSides;
    using Shape<T>::kRuns;
    int64_t tile, wave0, p0;
    int32_t strip, c;
    int lane, side, wave, run;
    bool live;

    // (false: there is nothing for this workgroup, which is one of those that round a grid up)
    template <int RUN>
    __device__ __forceinline__ bool take(const Scan &s, bool backward) {
        __shared__ uint32_t ticket;
        lane = threadIdx.x & (kLanes - 1);
        side = threadIdx.x / kLanes & (kSides - 1);
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        run = wave * kSides + side;
        uint32_t n = group_number();
        if (s.ticket) {
            // in the order in which workgroups come to life: one waits for none but those that live already
            if (threadIdx.x == 0) ticket = atomicAdd(s.ticket, 1u);
            __syncthreads();
            n = __builtin_amdgcn_readfirstlane(ticket);
        }
        tile = n / (uint32_t)s.strips;
        strip = (int32_t)(n - (uint32_t)tile * (uint32_t)s.strips);
        if (tile >= s.tiles) return false;
        if (backward) tile = s.tiles - 1 - tile;
        wave0 = tile * (kRuns * RUN) + wave * (kSides * RUN);
        p0 = wave0 + side * RUN;
        c = (strip * kLanes + lane) * V;
        live = c < s.width;
        c = live ? min(c, s.width - V) : 0;
        return true;
    }
    __device__ __forceinline__ uint64_t *word(const Scan &s, int64_t of) const { return s.words + ((of * s.strips + strip) * kLanes + lane) * V; }
};

template <typename T>
constexpr uint32_t kInfinite = sizeof(T) == 4 ? 0x7f800000u : std::is_same_v<T, bf16> ? 0x7f807f80u : 0x7c007c00u;

// A lane's run of a matrix's rows: what all lanes of the wavefront share of an address is kept in scalar registers, and a
// lane's own part in one.
template <typename T, int V, int RUN>
struct Run {
    static constexpr int kSides = Shape<T>::kSides;
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

// From the effects of a workgroup's runs (forward: in their order, backward: in the opposite one) to the state that enters
// each: they are joined inside the wavefronts, then over the tiles before, and applied from there.  What has to wait
// meanwhile waits in LDS: registers are full of rows.
template <typename T, int V, bool BACK>
struct Join {
    static constexpr int kLanes = Shape<T>::kLanes, kSides = Shape<T>::kSides;
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

    // The state that enters the tile: that which enters its group of tiles, and what the tiles of the group
    // before it do to it.  Each looking wavefront joins kLooks * kSides tiles, the first one joins what they found; a group's last
    // tile tells the state that enters the next group.  What is joined with what goes by a tile's number alone, never by
    // which state was known first, so that results are the same from call to call.
    __device__ __forceinline__ void behind(const Place<T, V> &p, const Scan &s, float (&state)[V]) {
        __shared__ Effect lds[kWaves][V][kLanes];
        __shared__ float lds_state[V][kLanes];
        const int64_t tile = BACK ? s.tiles - 1 - p.tile : p.tile;          // in the order of the chain
        const uint32_t size = (uint32_t)(s.lookers * kSides * kLooks), group = (uint32_t)tile / size;
        const int64_t first = (int64_t)group * size;
        const bool tells = p.run == 0 && p.live && tile + 1 < s.tiles, ends = tile + 1 == first + size;
        if (tells && !ends) {
#pragma unroll
            for (int k = 0; k < V; k++) publish(p.word(s, p.tile) + k, whole(p, k));
        }
        if (tile == 0) {
#pragma unroll
            for (int k = 0; k < V; k++) state[k] = 0.0f;
            return;
        }
        const bool asks = group > 0 && p.run == 0 && p.live;
        uint64_t w_group[V];
#pragma unroll
        for (int k = 0; k < V; k++) w_group[k] = asks ? look(p.word(s, s.tiles + group) + k) : 0;
        if (p.wave < s.lookers) {
            const int here = threadIdx.x & (kWave - 1);
            const uint64_t *at[kLooks];
            bool there[kLooks];
            uint64_t w[kLooks][V];
#pragma unroll
            for (int m = 0; m < kLooks; m++) {
                const int64_t of = tile - 1 - (p.run * kLooks + m);
                there[m] = of >= first && p.live;
                at[m] = p.word(s, there[m] ? BACK ? s.tiles - 1 - of : of : p.tile);
#pragma unroll
                for (int k = 0; k < V; k++) w[m][k] = there[m] ? look(at[m] + k) : 0;
            }
#pragma unroll
            for (int k = 0; k < V; k++) {
                Effect e = {1.0f, 0.0f};
#pragma unroll
                for (int m = 0; m < kLooks; m++) {
                    while (w[m][k] == kNotYet) w[m][k] = look(at[m] + k);
                    if (there[m]) e = then(effect_of(w[m][k]), e);
                }
#pragma unroll
                for (int d = 1; d < kSides; d <<= 1) {
                    const Effect o = {__shfl(e.A, here + d * kLanes), __shfl(e.H, here + d * kLanes)};
                    e = then(o, e);          // (of side 0, in the end, all sides)
                }
                if (p.side == 0) lds[p.wave][k][p.lane] = e;
            }
        }
        __syncthreads();
        if (p.run == 0) {
#pragma unroll
            for (int k = 0; k < V; k++) {
                Effect all = {1.0f, 0.0f};
                for (int q = 0; q < s.lookers; q++) all = then(lds[q][k][p.lane], all);
                while (w_group[k] == kNotYet) w_group[k] = look(p.word(s, s.tiles + group) + k);
                const float enters = asks ? all.of(effect_of(w_group[k]).H) : all.H;
                if (tells && ends) publish(p.word(s, s.tiles + group + 1) + k, {-1.0f, whole(p, k).of(enters)});
                lds_state[k][p.lane] = enters;
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < V; k++) state[k] = lds_state[k][p.lane];
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

// One tile.  INSIDE: of the inside of a sequence, the common case; else its wavefronts look for sequences' ends and for rows
// that are not there.
template <typename T, int V, int SPAN, bool STREAM, bool INSIDE>
__device__ __forceinline__ void scan(const Scan &s, const Place<T, V> &p, T *h, int64_t ldh, float *last, float *carry) {
    constexpr int RUN = SPAN / Shape<T>::kSides;
    const Sequences &seq = s.seq;
    const int32_t c = p.c;
    const int64_t left = seq.rows - p.p0;
    const int rows = INSIDE || left >= RUN ? RUN : left <= 0 ? 0 : (int)left;

    Raw<T, V> fr[RUN], xr[RUN];
    // (z is 0 where f is infinite: rows behind the last leave the state as it is)
    Run<T, V, RUN>(s.f, s.ldf, seq, p).load(fr, INSIDE, rows, kInfinite<T>);
    Run<T, V, RUN>(s.x, s.ldx, seq, p).load(xr, INSIDE, rows, 0u);
    Starts<RUN, Shape<T>::kSides> starts;
    if (!INSIDE) starts.find(seq, p.wave0, p.wave, p.side);
    float bias[V];
#pragma unroll
    for (int k = 0; k < V; k++) bias[k] = s.bias ? s.bias[c + k] * kLog2e : 0.0f;

    const uint64_t mine = (1ull << rows) - 1, firsts = INSIDE ? 0 : starts.first & mine, lasts = INSIDE ? 0 : starts.first >> 1 & mine;
    float state[V], A[V];
#pragma unroll
    for (int k = 0; k < V; k++) state[k] = 0.0f, A[k] = 1.0f;
#pragma unroll
        for (int i = 0; i < RUN; i++) {
            fr[i].renew();
            xr[i].renew();
            if (firsts >> i & 1) start_from<V>(state, s.h0, s.h0 ? starts.begun_by(seq, i) : 0, s.width, c);
#pragma unroll
            for (int k = 0; k < V; k++) {
                const float z = keep_not(fr[i][k], bias[k]);
                state[k] = next(z, state[k], xr[i][k]);
                A[k] = fmaf(-z, A[k], A[k]);
            }
        }
    Effect e[V];
#pragma unroll
    for (int k = 0; k < V; k++) e[k] = {firsts ? -1.0f : fmaxf(A[k], 0.0f), state[k]};
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
#pragma unroll
        for (int i = 0; i < RUN; i++) {
            fr[i].renew();
            xr[i].renew();
            if (firsts >> i & 1) start_from<V>(state, s.h0, s.h0 ? starts.begun_by(seq, i) : 0, s.width, c);
            Pack<T, V> out;
#pragma unroll
            for (int k = 0; k < V; k++) {
                state[k] = next(keep_not(fr[i][k], bias[k]), state[k], xr[i][k]);
                out.v[k] = (T)state[k];
            }
            if (p.live && i < rows) {
                store_pack<T, V>(to.row(i), out, STREAM);
                if (last && lasts >> i & 1) put<V>(last, starts.ended_by(seq, i), s.width, c, state);
            }
        }
}

template <typename T, int V, int SPAN, bool STREAM>
__global__ __launch_bounds__(kWaves *kWave, 4) void scan_kernel(Scan s, T *h, int64_t ldh, float *last, float *carry, int32_t *status) {
    constexpr int RUN = SPAN / Shape<T>::kSides, kRuns = Shape<T>::kRuns;
    Place<T, V> p;
    if (!p.template take<RUN>(s, false)) return;
    const Sequences &seq = s.seq;
    if (is_inside(seq, p.tile * (kRuns * RUN), kRuns * RUN)) scan<T, V, SPAN, STREAM, true>(s, p, h, ldh, last, carry);
    else scan<T, V, SPAN, STREAM, false>(s, p, h, ldh, last, carry);
    if (status && p.tile == 0 && p.strip == 0) check_sequences(seq, status);
    // a sequence without rows ends in the state that it begins with
    if (last && p.live && (seq.ptr || seq.each == 0)) {
        for (int64_t j = p.tile * kRuns + p.run; j < seq.count; j += s.tiles * kRuns) {
            if (seq.ptr && seq.ptr[j] < seq.ptr[j + 1]) continue;
#pragma unroll
            for (int k = 0; k < V; k++) last[j * s.width + p.c + k] = s.h0 ? s.h0[j * s.width + p.c + k] : 0.0f;
        }
    }
}

template <typename T>
struct Gradient {
    const T *dh;
    int64_t lddh;
    const float *dlast, *carry;
    T *df, *dx;
    int64_t lddf, lddx;
    float *dbias_part, *dh0;
};

template <typename T, int V, bool STREAM, bool INSIDE>
__device__ __forceinline__ void scan_backward(const Scan &s, const Gradient<T> &g, const Place<T, V> &p, float (&sum)[V]) {
    constexpr int RUN = Shape<T>::kBackwardRun, kRuns = Shape<T>::kRuns;
    static_assert(kRuns * RUN % CP_RECURRENCE_CHUNK == 0, "a tile begins where a state was kept");
    const Sequences &seq = s.seq;
    const int32_t c = p.c;
    const int64_t left = seq.rows - p.p0;
    const int rows = INSIDE || left >= RUN ? RUN : left <= 0 ? 0 : (int)left;

    Raw<T, V> fr[RUN], xr[RUN], dr[RUN];
    Run<T, V, RUN>(s.f, s.ldf, seq, p).load(fr, INSIDE, rows, kInfinite<T>);
    Run<T, V, RUN>(g.dh, g.lddh, seq, p).load(dr, INSIDE, rows, 0u);
    Run<T, V, RUN>(s.x, s.ldx, seq, p).load(xr, INSIDE, rows, 0u);
    float state[V], bias[V];
#pragma unroll
    for (int k = 0; k < V; k++) {
        bias[k] = s.bias ? s.bias[c + k] * kLog2e : 0.0f;
        // the state that enters the tile was kept
        state[k] = p.tile ? g.carry[p.tile * (kRuns * RUN / CP_RECURRENCE_CHUNK) * s.width + c + k] : 0.0f;
    }
    Starts<RUN, Shape<T>::kSides> starts;
    if (!INSIDE) starts.find(seq, p.wave0, p.wave, p.side);

    const uint64_t mine = (1ull << rows) - 1, firsts = INSIDE ? 0 : starts.first & mine, lasts = INSIDE ? 0 : starts.first >> 1 & mine;
    float z[RUN][V], u[V];               // (z's registers are the states' below)
    Effect e[V], d[V];
    {
        float run[V], A[V];
#pragma unroll
        for (int k = 0; k < V; k++) run[k] = 0.0f, A[k] = 1.0f, u[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < RUN; i++) {
                fr[i].renew();
                xr[i].renew();
                if (firsts >> i & 1) start_from<V>(run, s.h0, s.h0 ? starts.begun_by(seq, i) : 0, s.width, c);
#pragma unroll
                for (int k = 0; k < V; k++) {
                    z[i][k] = keep_not(fr[i][k], bias[k]);
                    run[k] = next(z[i][k], run[k], xr[i][k]);
                    A[k] = fmaf(-z[i][k], A[k], A[k]);
                }
                }
#pragma unroll
            for (int i = RUN - 1; i >= 0; i--) {
                dr[i].renew();
                if (lasts >> i & 1) start_from<V>(u, g.dlast, g.dlast ? starts.ended_by(seq, i) : 0, s.width, c);
#pragma unroll
                for (int k = 0; k < V; k++) {
                    const float to = u[k] + dr[i][k];
                    u[k] = fmaf(-z[i][k], to, to);
                }
            }
#pragma unroll
        for (int k = 0; k < V; k++) {
            const float a = fmaxf(A[k], 0.0f);
            e[k] = {firsts ? -1.0f : a, run[k]};
            d[k] = {lasts ? -1.0f : a, u[k]};
        }
    }
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
    float before[RUN][V];
#pragma unroll
    for (int k = 0; k < V; k++) sum[k] = 0.0f;
    const Run<T, V, RUN> to_f(g.df, g.lddf, seq, p), to_x(g.dx, g.lddx, seq, p);
#pragma unroll
        for (int i = 0; i < RUN; i++) {
            xr[i].renew();
            if (firsts >> i & 1) start_from<V>(state, s.h0, s.h0 ? starts.begun_by(seq, i) : 0, s.width, c);
#pragma unroll
            for (int k = 0; k < V; k++) {
                before[i][k] = state[k];
                state[k] = next(z[i][k], state[k], xr[i][k]);
            }
        }
#pragma unroll
        for (int i = RUN - 1; i >= 0; i--) {
            fr[i].renew();
            xr[i].renew();
            dr[i].renew();
            if (lasts >> i & 1) start_from<V>(u, g.dlast, g.dlast ? starts.ended_by(seq, i) : 0, s.width, c);
            Pack<T, V> of, ox;
#pragma unroll
            for (int k = 0; k < V; k++) {
                const float ef = odds(fr[i][k], bias[k]), z = fast_rcp(1.0f + ef);
                const float a = ef < 1.0f ? ef * z : 1.0f - z;      // (exact to its size at both ends)
                const float to = dr[i][k] + u[k], gz = to * z;
                const float v = gz * a * (before[i][k] - xr[i][k]);
                ox.v[k] = (T)gz;
                of.v[k] = (T)v;
                sum[k] += i < rows ? v : 0.0f;
                u[k] = to - gz;
            }
            if (p.live && i < rows) {
                store_pack<T, V>(to_x.row(i), ox, STREAM);
                store_pack<T, V>(to_f.row(i), of, STREAM);
                if (g.dh0 && firsts >> i & 1) put<V>(g.dh0, starts.begun_by(seq, i), s.width, c, u);
            }
        }
}

template <typename T, int V, bool STREAM>
__global__ __launch_bounds__(kWaves *kWave, 4) void scan_backward_kernel(Scan s, Gradient<T> g, int32_t *status) {
    constexpr int RUN = Shape<T>::kBackwardRun, kRuns = Shape<T>::kRuns, kLanes = Shape<T>::kLanes;
    Place<T, V> p;
    if (!p.template take<RUN>(s, true)) return;
    const Sequences &seq = s.seq;
    float sum[V];                        // of df over the lane's rows
    if (is_inside(seq, p.tile * (kRuns * RUN), kRuns * RUN)) scan_backward<T, V, STREAM, true>(s, g, p, sum);
    else scan_backward<T, V, STREAM, false>(s, g, p, sum);
    if (status && p.tile == s.tiles - 1 && p.strip == 0) check_sequences(seq, status);
    if (g.dbias_part) {
        __shared__ float lds[kWaves][V][kLanes];
#pragma unroll
        for (int k = 0; k < V; k++) {
#pragma unroll
            for (int off = kLanes; off < kWave; off <<= 1) sum[k] += __shfl_xor(sum[k], off);
            if (p.side == 0) lds[p.wave][k][p.lane] = sum[k];
        }
        __syncthreads();
        if (p.run == 0 && p.live) {
#pragma unroll
            for (int k = 0; k < V; k++) {
                float all = 0.0f;
                for (int w = 0; w < kWaves; w++) all += lds[w][k][p.lane];
                g.dbias_part[p.tile * s.width + p.c + k] = all;
            }
        }
    }
    if (g.dh0 && p.live && (seq.ptr || seq.each == 0)) {
        for (int64_t j = p.tile * kRuns + p.run; j < seq.count; j += s.tiles * kRuns) {
            if (seq.ptr && seq.ptr[j] < seq.ptr[j + 1]) continue;
#pragma unroll
            for (int k = 0; k < V; k++) g.dh0[j * s.width + p.c + k] = g.dlast ? g.dlast[j * s.width + p.c + k] : 0.0f;
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
                const float z = keep_not((float)fv.v[k], bias ? bias[c + k] * kLog2e : 0.0f);
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
    // (a workgroup's loops over the pointers count on by its threads, in 32 bits)
    if (seq_ptr ? num_seq > CP_RECURRENCE_MAX_PACKED : rows % num_seq != 0) return CP_ERR_SIZE;
    return CP_OK;
}

int64_t chunks_of(int64_t rows) { return (rows + CP_RECURRENCE_CHUNK - 1) / CP_RECURRENCE_CHUNK; }

int64_t tiles_of(int64_t rows, int span) {
    const int64_t tile = kWaves * span;
    return std::max<int64_t>(1, (rows + tile - 1) / tile);
}

// A ticket, and an effect for each tile and each group of two tiles or more, and channel, channels counted up to whole strips
// of the narrower types' lanes
int64_t words_of(int64_t tiles, int64_t group) { return tiles + (tiles + group - 1) / group; }
size_t words_bytes(int64_t rows, int32_t width, bool backward) {
    constexpr size_t strip = Shape<bf16>::kLanes * kWide;
    return kPolicyAlign + align_up(words_of(tiles_of(rows, backward ? kBackwardSpan : forward_span(rows, 2)), 2) * ((width + strip - 1) / strip * strip) * sizeof(uint64_t));
}
size_t part_bytes(int64_t rows, int32_t width) { return align_up((size_t)tiles_of(rows, kBackwardSpan) * width * sizeof(float)); }

// Wavefronts that look back, kLooks * kSides tiles each: a group.  The chain of states passes from group to group; the fewer strips
// there are, the more tiles of each are under way at once, and the faster it has to be.
int lookers_of(int32_t strips) { return std::max(1, std::min(kWaves, 32 / strips)); }

// Results that fill the caches go past them, unless neighbouring strips write parts of the same 32 bytes: 234037 x 411 bf16
// forward and backward take 597 us past the caches and 569 through them, 74241 x 1016 float 583 and 600.
bool past_caches(int64_t rows, int32_t width, size_t bytes, int results) {
    return results * (size_t)rows * width * bytes > kStreamed && width * bytes % 32 == 0;
}

void split_over(Scan &s, int span, int strip, void *workspace) {
    s.strips = (s.width + strip - 1) / strip;
    s.tiles = tiles_of(s.seq.rows, span);
    s.lookers = lookers_of(s.strips);
    s.ticket = s.tiles > 1 ? (uint32_t *)workspace : nullptr;
    s.words = s.tiles > 1 ? (uint64_t *)((char *)workspace + kPolicyAlign) : nullptr;
}

void clear_words(const Scan &s, int strip, int each, hipStream_t stream) {
    const int64_t count = words_of(s.tiles, s.lookers * each) * s.strips * strip;
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
    // (h in the place of an input is not possible: a strip of channels may read one of its neighbour's.  Nor is last in h0's: a sequence's
    // end may be known before its first tile has read its start a second time.)
    const auto matrix = [&](const void *at, int64_t ld) { return matrix_at(at, rows, width, ld, type); };
    const auto states = [&](const void *at) { return vector_at(at, (int64_t)num_seq * width); };
    if (in_the_way({matrix(f, ldf), matrix(x, ldx), vector_at(bias, width), states(h0)},
                   {matrix(h, ldh), states(last), vector_at(carry, chunks_of(rows) * width)}))
        return CP_ERR_ARG;
    if (rows < 2) ldf = ldx = ldh = width;         // (a single row is no distance from another)
    Scan s{};
    s.seq = {seq_ptr, rows, rows / num_seq, num_seq, reverse != 0};
    s.width = width;
    s.f = f, s.ldf = ldf, s.x = x, s.ldx = ldx, s.bias = bias, s.h0 = h0;
    const hipStream_t st = (hipStream_t)stream;
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        auto go = [&](auto v) {
            constexpr int V = decltype(v)::value;
            constexpr int strip = Shape<T>::kLanes * V;
            split_over(s, forward_span(rows, sizeof(T)), strip, workspace);
            const bool past = past_caches(rows, width, sizeof(T), 1);
            auto *kernel = past ? scan_kernel<T, V, kLongSpan, true> : scan_kernel<T, V, kLongSpan, false>;
            if constexpr (sizeof(T) == 2) {
                if (forward_span(rows, sizeof(T)) == kShortSpan)
                    kernel = past ? scan_kernel<T, V, kShortSpan, true> : scan_kernel<T, V, kShortSpan, false>;
            }
            if (s.tiles * s.strips > INT32_MAX) return (int)CP_ERR_SIZE;
            if (s.ticket) clear_words(s, strip, kLooks * Shape<T>::kSides, st);
            hipLaunchKernelGGL(kernel, grid_of(s.tiles * s.strips), dim3(kWaves * kWave), 0, st, s, (T *)h, ldh, last, carry,
                               seq_ptr ? status_out : nullptr);
            return launched();
        };
        if (width >= kWide) return go(std::integral_constant<int, kWide>{});
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
    const auto matrix = [&](const void *at, int64_t ld) { return matrix_at(at, rows, width, ld, type); };
    const auto states = [&](const void *at) { return vector_at(at, (int64_t)num_seq * width); };
    if (in_the_way({matrix(dh, lddh), matrix(f, ldf), matrix(x, ldx), states(dlast), states(h0), vector_at(bias, width),
                    vector_at(carry, chunks_of(rows) * width)},
                   {matrix(df, lddf), matrix(dx, lddx), states(dh0), vector_at(dbias, width)}))
        return CP_ERR_ARG;
    if (rows < 2) lddh = ldf = ldx = lddf = lddx = width;
    // (the sums of a single tile are the whole sums)
    const bool alone = tiles_of(rows, kBackwardSpan) == 1;
    float *part = !dbias || alone ? dbias : (float *)((char *)workspace + words_bytes(rows, width, true));
    Scan s{};
    s.seq = {seq_ptr, rows, rows / num_seq, num_seq, reverse != 0};
    s.width = width;
    s.f = f, s.ldf = ldf, s.x = x, s.ldx = ldx, s.bias = bias, s.h0 = h0;
    const hipStream_t st = (hipStream_t)stream;
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        auto go = [&](auto v) {
            constexpr int V = decltype(v)::value;
            constexpr int strip = Shape<T>::kLanes * V;
            split_over(s, kBackwardSpan, strip, workspace);
            auto *kernel = past_caches(rows, width, sizeof(T), 2) ? scan_backward_kernel<T, V, true> : scan_backward_kernel<T, V, false>;
            if (s.tiles * s.strips > INT32_MAX) return (int)CP_ERR_SIZE;
            if (s.ticket) clear_words(s, strip, kLooks * Shape<T>::kSides, st);
            hipLaunchKernelGGL(kernel, grid_of(s.tiles * s.strips), dim3(kWaves * kWave), 0, st, s,
                               Gradient<T>{(const T *)dh, lddh, dlast, carry, (T *)df, (T *)dx, lddf, lddx, part, dh0}, seq_ptr ? status_out : nullptr);
            if (dbias && !alone)
                hipLaunchKernelGGL(column_sum_kernel, dim3((width + 15) / 16), dim3(1024), 0, st, part, s.tiles, width, dbias);
            return launched();
        };
        if (width >= kWide) return go(std::integral_constant<int, kWide>{});
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
    const auto matrix = [&](const void *at, int64_t ld) { return matrix_at(at, num_seq, width, ld, type); };
    const Extent states = vector_at(state, (int64_t)num_slots * width);
    if (in_the_way({matrix(f, ldf), matrix(x, ldx)}, {matrix(h, ldh)}, true) ||
        in_the_way({matrix(f, ldf), matrix(x, ldx), vector_at(bias, width), vector_at(slots, num_seq, sizeof(int32_t))}, {states}) ||
        in_the_way({states, vector_at(bias, width), vector_at(slots, num_seq, sizeof(int32_t))}, {matrix(h, ldh)}))
        return CP_ERR_ARG;
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
        // (no two lanes may share a channel here: its state is read and written.  4096 x 2048 bf16 18.4 us, x 2047 25.9; float 27.2, 32.8)
        if (width % 4 == 0) return go(std::integral_constant<int, 4>{});
        return go(std::integral_constant<int, 1>{});
    });
}

}  // extern "C"
