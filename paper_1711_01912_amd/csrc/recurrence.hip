// Gated linear recurrence over rows of `width` channels, cut into sequences:
//
//   a = sigmoid(f + bias), z = 1 - a = sigmoid(-(f + bias)),  h_t = a_t h_{t-1} + z_t x_t
//
// z is formed directly, as 1 / (1 + e^(f + bias)), so that channels with a near 1 (long time scales) lose nothing.  A run of
// rows turns the state h that enters it into A h + H, with A the product of its a and H the state it ends in from zero: runs
// are taken by different wavefronts and joined.  Backward, with u_t = a_t g_t what flows into h_{t-1}:
//
//   g_t = dh_t + u_{t+1},  dx_t = z_t g_t,  df_t = g_t (h_{t-1} - x_t) a_t z_t,  u_t = a_t (dh_t + u_{t+1})
//
// the same kind of recurrence from the last row to the first; h_{t-1} is computed again from states kept every kChunk rows.
// Rows are counted in the direction of the scan throughout ("position"): of a reversed scan, position 0 is the last row.
// States, products and sums are floats; a row's result is rounded once, to the element type.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "policy.hpp"

namespace cpeval {

namespace {

constexpr int kWaves = 8;                    // wavefronts of a workgroup, one behind the other along the rows
constexpr int kRun = 16;                     // rows a wavefront holds in registers
constexpr int kChunk = kWaves * kRun;        // rows of a workgroup
static_assert(kChunk == CP_RECURRENCE_CHUNK, "the states kept for the backward pass enter every kChunk-th row");

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

    // how many sequences start at or before `position` (by a whole wavefront: 64 probes a round).  Bounded, and within the
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

    // the sequence (in scan order) that holds a position
    __device__ __forceinline__ int32_t at(int64_t position) const { return max(begun(position) - 1, 0); }

    // bit i: position p0 + i is the first of a sequence, or lies behind the last row; i = 0 .. kRun
    __device__ uint32_t firsts(int64_t p0) const {
        uint32_t bits = 0;
        if (!ptr) {
            for (int64_t s = each * (((uint32_t)p0 + (uint32_t)each - 1) / (uint32_t)each); s <= p0 + kRun && s < rows; s += each)
                bits |= 1u << (s - p0);
        } else {
            const int lane = threadIdx.x & (kWave - 1);
            for (int32_t j = p0 > 0 ? begun(p0 - 1) : 0; j < count; j += kWave) {
                const int64_t s = j + lane < count ? start(j + lane) : INT64_MAX;
                const bool in = s >= p0 && s <= p0 + kRun && s < rows;
                if (__ballot(in)) {
#pragma unroll
                    for (int i = 0; i <= kRun; i++) bits |= __ballot(in && s == p0 + i) ? 1u << i : 0u;
                }
                if (__ballot(s > p0 + kRun)) break;
            }
        }
        if (rows >= p0 && rows <= p0 + kRun) bits |= 1u << (rows - p0);
        return bits;
    }
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
    if (threadIdx.x == 0 && status) *status = bad ? CP_STATUS_BAD_SEQUENCE : CP_STATUS_OK;
}

// A run's effect on the state that enters it: h -> A h + H, or h -> H where a sequence begins inside (A < 0)
struct Effect {
    float A, H;
    __device__ __forceinline__ float of(float h) const { return A < 0 ? H : fmaf(A, h, H); }
};

__device__ __forceinline__ Effect then(Effect p, Effect q) {
    return q.A < 0 ? q : Effect{p.A < 0 ? p.A : p.A * q.A, fmaf(q.A, p.H, q.H)};
}

__device__ __forceinline__ float keep_not(float f, float bias) { return fast_rcp(1.0f + fast_exp(f + bias)); }   // z

// (1 - z) h + z x, with h - z h rounded once: 1 - z, rounded, would be off by more than z where z is small
__device__ __forceinline__ float next(float z, float h, float x) { return fmaf(z, x, fmaf(-z, h, h)); }

struct Scan {
    Sequences seq;
    int32_t width;
    const void *f, *x;
    int64_t ldf, ldx;
    const float *bias, *h0;
    float *carry;            // [chunks][width]: the state that enters each chunk
    Effect *effect;          // [chunks][width]: what each chunk does to it
};

template <typename T, int V>
struct Strip {
    int64_t c;               // the lane's first channel
    bool live;
    float bias[V];
    __device__ Strip(const Scan &s) {
        const int lane = threadIdx.x & (kWave - 1);
        c = ((int64_t)blockIdx.y * kWave + lane) * V;
        live = c < s.width;
        c = live ? c : 0;
#pragma unroll
        for (int k = 0; k < V; k++) bias[k] = s.bias ? s.bias[c + k] : 0.0f;
    }
};

// loads kRun rows from position p0 on; rows behind the last are the last one's
template <typename T, int V>
__device__ __forceinline__ void load_run(Pack<T, V> (&to)[kRun], const void *from, int64_t ld, int64_t c, const Sequences &seq,
                                         int64_t p0) {
#pragma unroll
    for (int i = 0; i < kRun; i++)
        to[i] = load_pack<T, V>((const T *)from + seq.row(min(p0 + i, seq.rows - 1)) * ld + c);
}

// MODE 0: the effect of every chunk.  MODE 1: h, from the states that enter the chunks.
template <typename T, int V, int MODE>
__global__ __launch_bounds__(kWaves *kWave) void scan_kernel(Scan s, T *h, int64_t ldh, float *last, int32_t *status) {
    __shared__ float lds_a[kWaves][V][kWave], lds_h[kWaves][V][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const Sequences &seq = s.seq;
    const int64_t chunk = blockIdx.x, p0 = chunk * kChunk + wave * kRun;
    const Strip<T, V> strip(s);
    const int64_t c = strip.c;
    const int rows = (int)min<int64_t>(max<int64_t>(seq.rows - p0, 0), kRun);

    Pack<T, V> fr[kRun], xr[kRun];
    if (rows > 0) {
        load_run<T, V>(fr, s.f, s.ldf, c, seq, p0);
        load_run<T, V>(xr, s.x, s.ldx, c, seq, p0);
    }
    const uint32_t first = rows > 0 ? seq.firsts(p0) : 0;
    if (MODE == 1 && status && blockIdx.x == 0 && blockIdx.y == 0) check_sequences(seq, status);

    float z[kRun][V];
    Effect e[V];
#pragma unroll
    for (int k = 0; k < V; k++) e[k] = {1.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kRun; i++)
        if (i < rows) {
            float start[V];
            const bool begins = first >> i & 1;
            if (begins) {
                const int32_t j = s.h0 ? seq.number(seq.at(p0 + i)) : 0;
#pragma unroll
                for (int k = 0; k < V; k++) start[k] = s.h0 ? s.h0[(int64_t)j * s.width + c + k] : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < V; k++) {
                z[i][k] = keep_not((float)fr[i].v[k], strip.bias[k]);
                if (begins) e[k] = {-1.0f, start[k]};
                e[k].H = next(z[i][k], e[k].H, (float)xr[i].v[k]);
                e[k].A = e[k].A < 0 ? e[k].A : fmaf(-z[i][k], e[k].A, e[k].A);
            }
        }
#pragma unroll
    for (int k = 0; k < V; k++) {
        lds_a[wave][k][lane] = e[k].A;
        lds_h[wave][k][lane] = e[k].H;
    }
    __syncthreads();
    if (MODE == 0) {
        if (wave == 0 && strip.live) {
#pragma unroll
            for (int k = 0; k < V; k++) {
                Effect all = {lds_a[0][k][lane], lds_h[0][k][lane]};
                for (int w = 1; w < kWaves; w++) all = then(all, {lds_a[w][k][lane], lds_h[w][k][lane]});
                s.effect[chunk * s.width + c + k] = all;
            }
        }
        return;
    }
    float state[V];
#pragma unroll
    for (int k = 0; k < V; k++) {
        state[k] = chunk ? s.carry[chunk * s.width + c + k] : 0.0f;
        for (int w = 0; w < wave; w++) state[k] = Effect{lds_a[w][k][lane], lds_h[w][k][lane]}.of(state[k]);
    }
#pragma unroll
    for (int i = 0; i < kRun; i++)
        if (i < rows) {
            if (first >> i & 1) {
                const int32_t j = s.h0 ? seq.number(seq.at(p0 + i)) : 0;
#pragma unroll
                for (int k = 0; k < V; k++) state[k] = s.h0 ? s.h0[(int64_t)j * s.width + c + k] : 0.0f;
            }
            Pack<T, V> out;
#pragma unroll
            for (int k = 0; k < V; k++) {
                state[k] = next(z[i][k], state[k], (float)xr[i].v[k]);
                out.v[k] = (T)state[k];
            }
            if (strip.live) store_pack<T, V>(h + seq.row(p0 + i) * ldh + c, out);
            if (last && (first >> (i + 1) & 1)) {
                const int32_t j = seq.number(seq.at(p0 + i));
                if (strip.live) {
#pragma unroll
                    for (int k = 0; k < V; k++) last[(int64_t)j * s.width + c + k] = state[k];
                }
            }
        }
    // a sequence without rows ends in the state that it begins with
    if (last) {
        for (int64_t j = chunk * kWaves + wave; j < seq.count; j += (int64_t)gridDim.x * kWaves) {
            const bool none = seq.ptr ? seq.ptr[j] >= seq.ptr[j + 1] : seq.each == 0;
            if (!none || !strip.live) continue;
#pragma unroll
            for (int k = 0; k < V; k++) last[j * s.width + c + k] = s.h0 ? s.h0[j * s.width + c + k] : 0.0f;
        }
    }
}

// the states that enter the chunks, one channel a lane; `from`, `step`: chunks in the order of the scan
__global__ __launch_bounds__(kWave) void carry_kernel(const Effect *effect, float *carry, int64_t chunks, int32_t width, bool back) {
    const int64_t c = (int64_t)blockIdx.x * kWave + threadIdx.x;
    if (c >= width) return;
    float h = 0.0f;
#pragma unroll 8
    for (int64_t i = 0; i < chunks; i++) {
        const int64_t at = (back ? chunks - 1 - i : i) * width + c;
        const Effect e = effect[at];
        carry[at] = h;
        h = e.of(h);
    }
}

// MODE 0: what every chunk does to the u that enters it from behind.  MODE 1: gradients.
template <typename T, int V, int MODE>
__global__ __launch_bounds__(kWaves *kWave) void scan_backward_kernel(Scan s, const T *dh, int64_t lddh, const float *dlast,
                                                                      const float *behind, T *df, int64_t lddf, T *dx, int64_t lddx,
                                                                      float *dbias_part, float *dh0, int32_t *status) {
    __shared__ float lds_a[kWaves][V][kWave], lds_h[kWaves][V][kWave], lds_u[kWaves][V][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const Sequences &seq = s.seq;
    const int64_t chunk = blockIdx.x, p0 = chunk * kChunk + wave * kRun;
    const Strip<T, V> strip(s);
    const int64_t c = strip.c;
    const int rows = (int)min<int64_t>(max<int64_t>(seq.rows - p0, 0), kRun);

    Pack<T, V> fr[kRun], xr[kRun], dr[kRun];
    if (rows > 0) {
        load_run<T, V>(fr, s.f, s.ldf, c, seq, p0);
        if (MODE == 1) load_run<T, V>(xr, s.x, s.ldx, c, seq, p0);
        load_run<T, V>(dr, dh, lddh, c, seq, p0);
    }
    const uint32_t first = rows > 0 ? seq.firsts(p0) : 0;
    if (MODE == 1 && status && blockIdx.x == 0 && blockIdx.y == 0) check_sequences(seq, status);

    float z[kRun][V], before[kRun][V];
    Effect e[V], ue[V];
#pragma unroll
    for (int k = 0; k < V; k++) e[k] = ue[k] = {1.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kRun; i++)
        if (i < rows) {
            const bool begins = first >> i & 1;
            float start[V];
            if (MODE == 1 && begins) {
                const int32_t j = s.h0 ? seq.number(seq.at(p0 + i)) : 0;
#pragma unroll
                for (int k = 0; k < V; k++) start[k] = s.h0 ? s.h0[(int64_t)j * s.width + c + k] : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < V; k++) {
                z[i][k] = keep_not((float)fr[i].v[k], strip.bias[k]);
                if (MODE == 1) {
                    if (begins) e[k] = {-1.0f, start[k]};
                    e[k].H = next(z[i][k], e[k].H, (float)xr[i].v[k]);
                    e[k].A = e[k].A < 0 ? e[k].A : fmaf(-z[i][k], e[k].A, e[k].A);
                }
            }
        }
#pragma unroll
    for (int i = kRun - 1; i >= 0; i--)
        if (i < rows) {
            const bool ends = first >> (i + 1) & 1;
            float start[V];
            if (ends) {
                const int32_t j = dlast ? seq.number(seq.at(p0 + i)) : 0;
#pragma unroll
                for (int k = 0; k < V; k++) start[k] = dlast ? dlast[(int64_t)j * s.width + c + k] : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < V; k++) {
                if (ends) ue[k] = {-1.0f, start[k]};
                const float g = ue[k].H + (float)dr[i].v[k];
                ue[k].H = fmaf(-z[i][k], g, g);
                ue[k].A = ue[k].A < 0 ? ue[k].A : fmaf(-z[i][k], ue[k].A, ue[k].A);
            }
        }
#pragma unroll
    for (int k = 0; k < V; k++) {
        lds_a[wave][k][lane] = ue[k].A;
        lds_u[wave][k][lane] = ue[k].H;
    }
    __syncthreads();
    if (MODE == 0) {
        if (wave == 0 && strip.live) {
#pragma unroll
            for (int k = 0; k < V; k++) {
                Effect all = {lds_a[kWaves - 1][k][lane], lds_u[kWaves - 1][k][lane]};
                for (int w = kWaves - 2; w >= 0; w--) all = then(all, {lds_a[w][k][lane], lds_u[w][k][lane]});
                s.effect[chunk * s.width + c + k] = all;
            }
        }
        return;
    }
    float u[V], state[V], sum[V];
#pragma unroll
    for (int k = 0; k < V; k++) {
        u[k] = behind ? behind[chunk * s.width + c + k] : 0.0f;
        for (int w = kWaves - 1; w > wave; w--) u[k] = Effect{lds_a[w][k][lane], lds_u[w][k][lane]}.of(u[k]);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < V; k++) {
        lds_a[wave][k][lane] = e[k].A;
        lds_h[wave][k][lane] = e[k].H;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < V; k++) {
        state[k] = chunk ? s.carry[chunk * s.width + c + k] : 0.0f;
        for (int w = 0; w < wave; w++) state[k] = Effect{lds_a[w][k][lane], lds_h[w][k][lane]}.of(state[k]);
        sum[k] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kRun; i++)
        if (i < rows) {
            if (first >> i & 1) {
                const int32_t j = s.h0 ? seq.number(seq.at(p0 + i)) : 0;
#pragma unroll
                for (int k = 0; k < V; k++) state[k] = s.h0 ? s.h0[(int64_t)j * s.width + c + k] : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < V; k++) {
                before[i][k] = state[k];
                state[k] = next(z[i][k], state[k], (float)xr[i].v[k]);
            }
        }
#pragma unroll
    for (int i = kRun - 1; i >= 0; i--)
        if (i < rows) {
            if (first >> (i + 1) & 1) {
                const int32_t j = dlast ? seq.number(seq.at(p0 + i)) : 0;
#pragma unroll
                for (int k = 0; k < V; k++) u[k] = dlast ? dlast[(int64_t)j * s.width + c + k] : 0.0f;
            }
            Pack<T, V> of, ox;
#pragma unroll
            for (int k = 0; k < V; k++) {
                const float g = (float)dr[i].v[k] + u[k], gz = g * z[i][k], e = fast_exp((float)fr[i].v[k] + strip.bias[k]);
                const float a = e < 1.0f ? e * z[i][k] : 1.0f - z[i][k];      // (exact to its size at both ends)
                const float d = gz * a * (before[i][k] - (float)xr[i].v[k]);
                ox.v[k] = (T)gz;
                of.v[k] = (T)d;
                sum[k] += d;
                u[k] = g - gz;
            }
            const int64_t row = seq.row(p0 + i);
            if (strip.live) {
                store_pack<T, V>(dx + row * lddx + c, ox);
                store_pack<T, V>(df + row * lddf + c, of);
            }
            if (dh0 && (first >> i & 1)) {
                const int32_t j = seq.number(seq.at(p0 + i));
                if (strip.live) {
#pragma unroll
                    for (int k = 0; k < V; k++) dh0[(int64_t)j * s.width + c + k] = u[k];
                }
            }
        }
    if (dbias_part) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < V; k++) lds_u[wave][k][lane] = sum[k];
        __syncthreads();
        if (wave == 0 && strip.live) {
#pragma unroll
            for (int k = 0; k < V; k++) {
                float all = 0.0f;
                for (int w = 0; w < kWaves; w++) all += lds_u[w][k][lane];
                dbias_part[chunk * s.width + c + k] = all;
            }
        }
    }
    if (dh0) {
        for (int64_t j = chunk * kWaves + wave; j < seq.count; j += (int64_t)gridDim.x * kWaves) {
            const bool none = seq.ptr ? seq.ptr[j] >= seq.ptr[j + 1] : seq.each == 0;
            if (!none || !strip.live) continue;
#pragma unroll
            for (int k = 0; k < V; k++) dh0[j * s.width + c + k] = dlast ? dlast[j * s.width + c + k] : 0.0f;
        }
    }
}

// sums over rows of float partial sums, one column a lane, in a fixed order and in 64 bits
__global__ __launch_bounds__(256) void column_sum_kernel(const float *part, int64_t rows, int32_t width, float *out) {
    __shared__ double lds[4][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t c = (int64_t)blockIdx.x * kWave + lane;
    double sum = 0.0;
    if (c < width)
        for (int64_t i = wave; i < rows; i += 4) sum += part[i * width + c];
    lds[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && c < width) out[c] = (float)(((lds[0][lane] + lds[1][lane]) + lds[2][lane]) + lds[3][lane]);
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

int64_t chunks_of(int64_t rows) { return std::max<int64_t>(1, (rows + kChunk - 1) / kChunk); }

// V channels may be loaded at once: their number, the rows' distances and the addresses are multiples of it
bool fits(int v, size_t bytes, int32_t width, std::initializer_list<const void *> at, std::initializer_list<int64_t> ld) {
    if (width % v) return false;
    for (const void *p : at)
        if ((uintptr_t)p % (v * bytes)) return false;
    for (int64_t d : ld)
        if (d % v) return false;
    return true;
}

int check_scan(int64_t rows, int32_t width, int32_t num_seq, const int32_t *seq_ptr, int type, int reverse) {
    if (!known_type(type) || (reverse != 0 && reverse != 1)) return CP_ERR_ARG;
    if (rows < 0 || rows > INT32_MAX || width < 1 || width > CP_RECURRENCE_MAX_WIDTH || num_seq < 1) return CP_ERR_SIZE;
    if (!seq_ptr && rows % num_seq) return CP_ERR_SIZE;
    return CP_OK;
}

size_t work_bytes(int64_t rows, int32_t width) { return align_up((size_t)chunks_of(rows) * width * sizeof(Effect)); }
size_t part_bytes(int64_t rows, int32_t width) { return align_up((size_t)chunks_of(rows) * width * sizeof(float)); }

}  // namespace

}  // namespace cpeval

using namespace cpeval;

extern "C" {

int cp_recurrence_workspace_bytes(int64_t rows, int32_t width, int backward, size_t *out_bytes) {
    if (!out_bytes) return CP_ERR_NULL;
    if (rows < 0 || rows > INT32_MAX || width < 1 || width > CP_RECURRENCE_MAX_WIDTH) return CP_ERR_SIZE;
    *out_bytes = work_bytes(rows, width) + (backward ? 2 : 1) * part_bytes(rows, width);
    return CP_OK;
}

int cp_recurrence(int64_t rows, int32_t width, int32_t num_seq, const int32_t *seq_ptr, int type, int reverse, const void *f,
                  int64_t ldf, const void *x, int64_t ldx, const float *bias, const float *h0, void *h, int64_t ldh, float *last,
                  float *carry, void *workspace, size_t workspace_bytes, void *stream, int32_t *status_out) {
    int rc = check_scan(rows, width, num_seq, seq_ptr, type, reverse);
    if (rc) return rc;
    if ((rows > 0 && (!f || !x || !h)) || (seq_ptr && !status_out)) return CP_ERR_NULL;
    if (rows > 1 && (ldf < width || ldx < width || ldh < width)) return CP_ERR_SIZE;
    const int64_t chunks = chunks_of(rows);
    const bool split = chunks > 1;
    if (split) {
        if (!workspace) return CP_ERR_NULL;
        if ((uintptr_t)workspace % kPolicyAlign || workspace_bytes < work_bytes(rows, width) + part_bytes(rows, width)) return CP_ERR_WORKSPACE;
    }
    Scan s{{seq_ptr, rows, rows / num_seq, num_seq, reverse != 0}, width, f, x, ldf, ldx, bias, h0, carry, (Effect *)workspace};
    if (split && !carry) s.carry = (float *)((char *)workspace + work_bytes(rows, width));
    const hipStream_t st = (hipStream_t)stream;
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        auto go = [&](auto v) {
            constexpr int V = decltype(v)::value;
            const dim3 grid((unsigned)chunks, (unsigned)((width + kWave * V - 1) / (kWave * V)));
            if (split) {
                hipLaunchKernelGGL((scan_kernel<T, V, 0>), grid, dim3(kWaves * kWave), 0, st, s, (T *)h, ldh, last, status_out);
                hipLaunchKernelGGL(carry_kernel, dim3((width + kWave - 1) / kWave), dim3(kWave), 0, st, s.effect, s.carry, chunks, width, false);
            }
            hipLaunchKernelGGL((scan_kernel<T, V, 1>), grid, dim3(kWaves * kWave), 0, st, s, (T *)h, ldh, last, status_out);
            return launched();
        };
        // (four bytes a lane and row)
        constexpr int most = 4 / sizeof(T);
        if (most > 1 && fits(most, sizeof(T), width, {f, x, h}, {ldf, ldx, ldh})) return go(std::integral_constant<int, most>{});
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
    if (rows > 1 && (lddh < width || ldf < width || ldx < width || lddf < width || lddx < width)) return CP_ERR_SIZE;
    const int64_t chunks = chunks_of(rows);
    const bool split = chunks > 1;
    if (split && !carry) return CP_ERR_NULL;
    if (split || dbias) {
        if (!workspace) return CP_ERR_NULL;
        if ((uintptr_t)workspace % kPolicyAlign || workspace_bytes < work_bytes(rows, width) + 2 * part_bytes(rows, width)) return CP_ERR_WORKSPACE;
    }
    char *work = (char *)workspace;
    float *behind = split ? (float *)(work + work_bytes(rows, width)) : nullptr;
    float *part = dbias ? (float *)(work + work_bytes(rows, width) + part_bytes(rows, width)) : nullptr;
    Scan s{{seq_ptr, rows, rows / num_seq, num_seq, reverse != 0}, width, f, x, ldf, ldx, bias, h0, (float *)carry, (Effect *)work};
    const hipStream_t st = (hipStream_t)stream;
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        auto go = [&](auto v) {
            constexpr int V = decltype(v)::value;
            const dim3 grid((unsigned)chunks, (unsigned)((width + kWave * V - 1) / (kWave * V)));
            if (split) {
                hipLaunchKernelGGL((scan_backward_kernel<T, V, 0>), grid, dim3(kWaves * kWave), 0, st, s, (const T *)dh, lddh, dlast, behind, (T *)df,
                                   lddf, (T *)dx, lddx, part, dh0, status_out);
                hipLaunchKernelGGL(carry_kernel, dim3((width + kWave - 1) / kWave), dim3(kWave), 0, st, s.effect, behind, chunks, width, true);
            }
            hipLaunchKernelGGL((scan_backward_kernel<T, V, 1>), grid, dim3(kWaves * kWave), 0, st, s, (const T *)dh, lddh, dlast, behind, (T *)df, lddf,
                               (T *)dx, lddx, part, dh0, status_out);
            if (dbias)
                hipLaunchKernelGGL(column_sum_kernel, dim3((width + kWave - 1) / kWave), dim3(256), 0, st, part, rows > 0 ? chunks : 0, width, dbias);
            return launched();
        };
        constexpr int most = 4 / sizeof(T);
        if (most > 1 && fits(most, sizeof(T), width, {dh, f, x, df, dx}, {lddh, ldf, ldx, lddf, lddx})) return go(std::integral_constant<int, most>{});
        return go(std::integral_constant<int, 1>{});
    });
}

int cp_recurrence_step(int32_t num_seq, int32_t width, int type, const void *f, int64_t ldf, const void *x, int64_t ldx,
                       const float *bias, float *state, int32_t num_slots, const int32_t *slots, void *h, int64_t ldh, void *stream,
                       int32_t *status_out) {
    if (!known_type(type)) return CP_ERR_ARG;
    if (num_seq < 0 || num_slots < 1 || width < 1 || width > CP_RECURRENCE_MAX_WIDTH || (!slots && num_seq > num_slots)) return CP_ERR_SIZE;
    if ((num_seq > 0 && (!f || !x || !h)) || !state || (slots && !status_out)) return CP_ERR_NULL;
    if (num_seq > 1 && (ldf < width || ldx < width || ldh < width)) return CP_ERR_SIZE;
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
        if (fits(4, sizeof(T), width, {f, x, h}, {ldf, ldx, ldh}) && (uintptr_t)state % 16 == 0) return go(std::integral_constant<int, 4>{});
        return go(std::integral_constant<int, 1>{});
    });
}

}  // extern "C"
