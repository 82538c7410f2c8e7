// The joint between two blocks of a sequence model, in one pass over its rows:
//
//   u = y / rms(y) * w_post  (y itself without w_post),   r = x + scale * act(gate) * u,   z = r / rms(r) * w_pre
//
// with rms(v) = sqrt(mean(v^2) + eps), and its gradient.  z is formed from r in 32 bits, not from r as it is stored, and the
// backward pass computes r again from x, y and gate, which costs the reads that keeping r would.  With q = dr + what flows
// back through the second norm:
//
//   dx = q,  du = q scale act(gate),  dgate = q scale u act'(gate),  dw_pre = sum dz r/rms(r),  dw_post = sum du y/rms(y)
//
// Bound by memory: a row is held in registers by one workgroup, the smallest that has room for it at 16 bytes a load, so
// that every input is read once and every output written once.  Workgroups go over many rows: weights stay in registers, and
// so do the sums of the weights' gradients, which are joined over the workgroups at the end, in a fixed order.  Sums are
// floats (the weights' gradients' over a workgroup's rows; over workgroups they are of 64 bits); a result is rounded once, to its
// type.
// 32768 x 2048 bf16: 140 us forward (4.8 TB/s), 210 us backward (5.1 TB/s: the rate of a copy) and 7 us for the weights' sums.
// Backward rows of more than 8,192 values do not fit: 16 a thread and their products spill up to 73 registers a lane, and the weights are
// loaded twice a row.  4096 x 16384 bf16 455 us (209 at the rate of a copy), float 725 (419); 4096 x 8192 137 and 217 (105, 209).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "policy.hpp"

namespace cpeval {

namespace {

struct Joint {
    int64_t rows;
    int32_t width;
    const void *x, *y, *gate;
    int64_t ldx, ldy, ldg;
    const void *w_pre, *w_post;
    int weight_type, act;
    float scale, eps;
    float *stats;            // [2][rows]: 1 / rms of y and of r
};

// Rows: NT threads take one at a time.  Of NT below a wavefront's 64 lanes several rows lie side by side in a workgroup, which
// is one wavefront: 405303 rows of 70 fp16 values, 9 of 64 lanes having some, took 397 us forward and backward.
template <int NT>
struct Sharing {
    static constexpr int kSide = NT < kWave ? kWave / NT : 1, kThreads = NT < kWave ? kWave : NT;
    static __device__ __forceinline__ int thread() { return NT < kWave ? threadIdx.x & (NT - 1) : threadIdx.x; }
    static __device__ __forceinline__ int64_t first() { return NT < kWave ? (int64_t)blockIdx.x * kSide + threadIdx.x / NT : blockIdx.x; }
    static __device__ __forceinline__ int64_t step() { return (int64_t)gridDim.x * kSide; }
};

// Where a thread's values lie: NV vectors of V.  The last vector of a row that is no multiple of V is the row's last V
// values; those that are another vector's are `skip`ped in sums (and written twice, to the same).
template <int NT, int V, int NV>
struct Columns {
    int32_t c[NV], skip[NV];
    bool live[NV];
    __device__ __forceinline__ Columns(int32_t width) {
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int32_t first = (i * NT + Sharing<NT>::thread()) * V;
            live[i] = first < width;
            c[i] = live[i] ? min(first, width - V) : 0;
            skip[i] = live[i] ? first - c[i] : V;
        }
    }
};

// V weights as floats
template <int V>
__device__ __forceinline__ void load_weights(float (&to)[V], const void *w, int type, int32_t c) {
    auto from = [&](auto t) {
        using T = decltype(t);
        const Pack<T, V> p = load_pack<T, V>((const T *)w + c);
#pragma unroll
        for (int k = 0; k < V; k++) to[k] = (float)p.v[k];
    };
    if (type == CP_TYPE_F32) from(float{});
    else if (type == CP_TYPE_BF16) from(bf16{});
    else from(f16{});
}

// Sum over a row's threads, in every one of them.  `slot`: no two sums between which no other lies may have the same (a slow wavefront
// may still read what the last one left).
template <int NT>
__device__ __forceinline__ float group_sum(float v, int slot) {
    if constexpr (NT < kWave) {
#pragma unroll
        for (int off = NT / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
        return v;
    }
    v = wave_sum(v);
    if constexpr (NT > kWave) {
        __shared__ float lds[4][NT / kWave];
        if ((threadIdx.x & (kWave - 1)) == 0) lds[slot][threadIdx.x / kWave] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < NT / kWave; w++) v += lds[slot][w];
    }
    return v;
}

// act(gate) and its slope
__device__ __forceinline__ void gate_of(float g, int act, float &value, float &slope) {
    if (act == CP_GATE_NONE) {
        value = g;
        slope = 1.0f;
        return;
    }
    const float sg = fast_rcp(1.0f + fast_exp(-g));
    value = act == CP_GATE_SIGMOID ? sg : g * sg;
    slope = act == CP_GATE_SIGMOID ? sg * (1.0f - sg) : sg * (1.0f + g * (1.0f - sg));
}

// TS: the stream's type (x, r, dx, dr), TB: the block's (y, gate, z and their gradients)
template <typename TS, typename TB, int NT, int V, int NV>
__global__ __launch_bounds__(Sharing<NT>::kThreads) void joint_kernel(Joint j, TS *r_out, int64_t ldr, TB *z_out, int64_t ldz) {
    const Columns<NT, V, NV> at(j.width);
    const float inv = 1.0f / j.width;
    float w_pre[NV][V], w_post[NV][V];
#pragma unroll
    for (int i = 0; i < NV; i++) {
        load_weights<V>(w_pre[i], j.w_pre, j.weight_type, at.c[i]);
        if (j.w_post) load_weights<V>(w_post[i], j.w_post, j.weight_type, at.c[i]);
        else
#pragma unroll
            for (int k = 0; k < V; k++) w_post[i][k] = 1.0f;
    }
    // r in the place of an input: the row's last vector, moved back, reads what its neighbour is to write (z comes after a sum over
    // the row's threads, and so does r where there is one of y's)
    const bool over = r_out && (r_out == j.x || (const void *)r_out == j.y || (const void *)r_out == j.gate);
    int slot = 0;
    for (int64_t row = Sharing<NT>::first(); row < j.rows; row += Sharing<NT>::step(), slot ^= 2) {
        Raw<TS, V> x[NV];
        Raw<TB, V> y[NV], g[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) {
            if (j.y) y[i].load((const TB *)j.y + row * j.ldy + at.c[i]);
            x[i].load((const TS *)j.x + row * j.ldx + at.c[i]);
            if (j.gate) g[i].load((const TB *)j.gate + row * j.ldg + at.c[i]);
        }
        float ry = 1.0f;
        if (j.w_post) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; i++)
#pragma unroll
                for (int k = 0; k < V; k++) sum = k >= at.skip[i] ? fmaf(y[i][k], y[i][k], sum) : sum;
            ry = 1.0f / sqrtf(group_sum<NT>(sum, slot) * inv + j.eps);
        } else if (NT > kWave && over) {
            __syncthreads();
        }
        float r[NV][V], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            Pack<TS, V> out;
#pragma unroll
            for (int k = 0; k < V; k++) {
                r[i][k] = x[i][k];
                if (j.y) {
                    float value = 1.0f, slope;
                    if (j.gate) gate_of(g[i][k], j.act, value, slope);
                    r[i][k] = fmaf(j.scale * value, y[i][k] * ry * w_post[i][k], r[i][k]);
                }
                out.v[k] = (TS)r[i][k];
                sum = k >= at.skip[i] ? fmaf(r[i][k], r[i][k], sum) : sum;
            }
            if (r_out && at.live[i]) store_pack<TS, V>(r_out + row * ldr + at.c[i], out);
        }
        const float rr = 1.0f / sqrtf(group_sum<NT>(sum, slot + 1) * inv + j.eps);
#pragma unroll
        for (int i = 0; i < NV; i++) {
            Pack<TB, V> out;
#pragma unroll
            for (int k = 0; k < V; k++) out.v[k] = (TB)(r[i][k] * rr * w_pre[i][k]);
            if (at.live[i]) store_pack<TB, V>(z_out + row * ldz + at.c[i], out);
        }
        if (j.stats && Sharing<NT>::thread() == 0) {
            j.stats[row] = ry;
            j.stats[j.rows + row] = rr;
        }
    }
}

template <typename TS, typename TB>
struct JointGrad {
    const TS *dr;
    const TB *dz;
    TS *dx;
    TB *dy, *dg;
    int64_t lddr, lddz, lddx, lddy, lddg;
    float *part_pre, *part_post;         // [workgroups][width]
};

template <typename TS, typename TB, int NT, int V, int NV>
__global__ __launch_bounds__(Sharing<NT>::kThreads) void joint_backward_kernel(Joint j, JointGrad<TS, TB> b) {
    const Columns<NT, V, NV> at(j.width);
    const float inv = 1.0f / j.width;
    // (the longest rows leave no registers for weights and sums: these are kept in LDS, those loaded again for every row)
    constexpr bool APART = NV * V > 8;
    extern __shared__ float lds_acc[];               // APART: [2][NV * V][NT]
    float w_pre[NV][V], w_post[NV][V], acc_pre[NV][V], acc_post[NV][V];
    auto weights = [&](int i) {
        load_weights<V>(w_pre[i], j.w_pre, j.weight_type, at.c[i]);
        if (j.w_post) load_weights<V>(w_post[i], j.w_post, j.weight_type, at.c[i]);
        else
#pragma unroll
            for (int k = 0; k < V; k++) w_post[i][k] = 1.0f;
    };
    auto pre = [&](int i, int k) -> float & { return APART ? lds_acc[(i * V + k) * NT + threadIdx.x] : acc_pre[i][k]; };
    auto post = [&](int i, int k) -> float & { return APART ? lds_acc[((NV + i) * V + k) * NT + threadIdx.x] : acc_post[i][k]; };
#pragma unroll
    for (int i = 0; i < NV; i++) {
        if (!APART) weights(i);
#pragma unroll
        for (int k = 0; k < V; k++) pre(i, k) = post(i, k) = 0.0f;
    }
    int slot = 0;
    for (int64_t row = Sharing<NT>::first(); row < j.rows; row += Sharing<NT>::step(), slot ^= 2) {
        const float ry = j.w_post ? j.stats[row] : 1.0f, rr = j.stats[j.rows + row];
        Raw<TS, V> x[NV], d[NV];
        Raw<TB, V> y[NV], g[NV], e[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) {
            if (j.y) y[i].load((const TB *)j.y + row * j.ldy + at.c[i]);
            x[i].load((const TS *)j.x + row * j.ldx + at.c[i]);
            if (j.gate) g[i].load((const TB *)j.gate + row * j.ldg + at.c[i]);
            e[i].load(b.dz + row * b.lddz + at.c[i]);
            if (b.dr) d[i].load(b.dr + row * b.lddr + at.c[i]);
            else d[i].fill(0);
        }
        float rh[NV][V], dot = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            if (APART) weights(i);
#pragma unroll
            for (int k = 0; k < V; k++) {
                float r = x[i][k];
                if (j.y) {
                    float value = 1.0f, slope;
                    if (j.gate) gate_of(g[i][k], j.act, value, slope);
                    r = fmaf(j.scale * value, y[i][k] * ry * w_post[i][k], r);
                }
                rh[i][k] = r * rr;
                pre(i, k) = fmaf(e[i][k], rh[i][k], pre(i, k));
                dot = k >= at.skip[i] ? fmaf(e[i][k] * w_pre[i][k], rh[i][k], dot) : dot;
            }
        }
        dot = group_sum<NT>(dot, slot) * inv;
        float du[NV][V], dot2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            Pack<TS, V> ox;
            Pack<TB, V> og;
            if (APART) weights(i);
#pragma unroll
            for (int k = 0; k < V; k++) {
                const float q = fmaf(rr, fmaf(-rh[i][k], dot, e[i][k] * w_pre[i][k]), d[i][k]);
                ox.v[k] = (TS)q;
                if (j.y) {
                    float value = 1.0f, slope = 0.0f;
                    if (j.gate) gate_of(g[i][k], j.act, value, slope);
                    const float yh = y[i][k] * ry, qs = q * j.scale, dv = qs * value;
                    og.v[k] = (TB)(qs * yh * w_post[i][k] * slope);
                    post(i, k) = fmaf(dv, yh, post(i, k));
                    du[i][k] = dv * w_post[i][k];
                    dot2 = k >= at.skip[i] ? fmaf(du[i][k], yh, dot2) : dot2;
                }
            }
            if (at.live[i]) {
                store_pack<TS, V>(b.dx + row * b.lddx + at.c[i], ox);
                if (b.dg) store_pack<TB, V>(b.dg + row * b.lddg + at.c[i], og);
            }
        }
        if (!j.y) continue;
        if (j.w_post) dot2 = group_sum<NT>(dot2, slot + 1) * inv;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            Pack<TB, V> oy;
#pragma unroll
            for (int k = 0; k < V; k++) oy.v[k] = (TB)(j.w_post ? ry * fmaf(-y[i][k] * ry, dot2, du[i][k]) : du[i][k]);
            if (at.live[i]) store_pack<TB, V>(b.dy + row * b.lddy + at.c[i], oy);
        }
    }
    if constexpr (NT < kWave) {          // the rows side by side
#pragma unroll
        for (int k = 0; k < V; k++)
#pragma unroll
            for (int off = NT; off < kWave; off <<= 1) {
                pre(0, k) += __shfl_xor(pre(0, k), off);
                post(0, k) += __shfl_xor(post(0, k), off);
            }
        if (threadIdx.x >= NT) return;
    }
#pragma unroll
    for (int i = 0; i < NV; i++) {
        if (!at.live[i]) continue;
        const int64_t to = (int64_t)blockIdx.x * j.width + at.c[i];
#pragma unroll
        for (int k = 0; k < V; k++) {
            if (k < at.skip[i]) continue;            // (their owner has summed them too)
            if (b.part_pre) b.part_pre[to + k] = pre(i, k);
            if (b.part_post) b.part_post[to + k] = post(i, k);
        }
    }
}

// The weights' gradients from the workgroups' sums, 16 columns a workgroup, in a fixed order and in 64 bits
struct WeightSum {
    const float *part;
    void *out;
};
__global__ __launch_bounds__(1024) void weight_sum_kernel(WeightSum pre, WeightSum post, int32_t groups, int32_t width, int type) {
    __shared__ double lds[64][16];
    const WeightSum &w = blockIdx.y ? post : pre;
    const int lane = threadIdx.x & 15, first = threadIdx.x / 16;
    const int32_t c = blockIdx.x * 16 + lane;
    double sum = 0.0;
    if (c < width) {
#pragma unroll 4
        for (int32_t i = first; i < groups; i += 64) sum += w.part[(int64_t)i * width + c];
    }
    lds[first][lane] = sum;
    __syncthreads();
    if (first != 0 || c >= width) return;
    for (int i = 1; i < 64; i++) sum += lds[i][lane];
    if (type == CP_TYPE_F32) ((float *)w.out)[c] = (float)sum;
    else if (type == CP_TYPE_BF16) ((bf16 *)w.out)[c] = (bf16)(float)sum;
    else ((f16 *)w.out)[c] = (f16)(float)sum;
}

constexpr int kMostWaves = 16 * 256;         // that go over rows at once: what registers leave room for on 256 compute units

// Calls f(threads, values a load, loads a thread) for the fewest threads that hold a row.  16 bytes a load, of the wider
// of the two types; a thread holds at most 16 values, so that a workgroup's registers leave room for others.
template <int WIDE, typename F>
int by_shape(int32_t width, F f) {
    using std::integral_constant;
    if (width < WIDE) return f(integral_constant<int, 8>{}, integral_constant<int, 1>{}, integral_constant<int, 1>{});
    auto go = [&](auto nt, auto nv) { return f(nt, integral_constant<int, WIDE>{}, nv); };
    auto one = integral_constant<int, 1>{};
    if (width <= 8 * WIDE) return go(integral_constant<int, 8>{}, one);
    if (width <= 16 * WIDE) return go(integral_constant<int, 16>{}, one);
    if (width <= 32 * WIDE) return go(integral_constant<int, 32>{}, one);
    if (width <= 64 * WIDE) return go(integral_constant<int, 64>{}, one);
    if (width <= 128 * WIDE) return go(integral_constant<int, 128>{}, one);
    if (width <= 256 * WIDE) return go(integral_constant<int, 256>{}, one);
    if (width <= 512 * WIDE) return go(integral_constant<int, 512>{}, one);
    if (width <= 1024 * WIDE) return go(integral_constant<int, 1024>{}, one);
    if (width <= 2048 * WIDE) return go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
    if constexpr (2048 * WIDE < CP_NORM_MAX_WIDTH) return go(integral_constant<int, 1024>{}, integral_constant<int, 16 / WIDE>{});
    return (int)CP_ERR_SIZE;
}
static_assert(1024 * 16 >= CP_NORM_MAX_WIDTH, "the largest workgroup holds the longest row");

// Workgroups that go over rows.  (Threads of a row: as by_shape takes them.)
int groups_of(int64_t rows, int32_t width, int wide) {
    int nt = 8;
    while (nt < 1024 && width > nt * wide) nt *= 2;
    if (nt < kWave) return (int)std::min<int64_t>((rows + kWave / nt - 1) / (kWave / nt), kMostWaves);
    return (int)std::min<int64_t>(rows, kMostWaves / (nt / kWave));
}

// a workspace's half: the sums of as many workgroups as any pair of types makes
size_t part_bytes(int64_t rows, int32_t width) {
    return align_up((size_t)std::max(groups_of(rows, width, 8), groups_of(rows, width, 4)) * width * sizeof(float));
}

int check_joint(int64_t rows, int32_t width, int stream_type, int type, int weight_type, int act) {
    if (!known_type(stream_type) || !known_type(type) || !known_type(weight_type)) return CP_ERR_ARG;
    if ((stream_type != type && stream_type != CP_TYPE_F32) || act < CP_GATE_NONE || act > CP_GATE_SILU) return CP_ERR_ARG;
    if (rows < 0 || width < 1 || width > CP_NORM_MAX_WIDTH) return CP_ERR_SIZE;
    return CP_OK;
}

// the pairs of element types: the stream as the block, or in 32 bits
template <typename F>
int by_types(int stream_type, int type, F f) {
    return by_type(type, [&](auto t) {
        using TB = decltype(t);
        return stream_type == type ? f(TB{}, TB{}) : f(float{}, TB{});
    });
}

}  // namespace

}  // namespace cpeval

using namespace cpeval;

extern "C" {

int cp_norm_gate(int64_t rows, int32_t width, int stream_type, int type, int weight_type, int gate_act, const void *x, int64_t ldx,
                 const void *y, int64_t ldy, const void *gate, int64_t ldg, const void *w_pre, const void *w_post, float scale, float eps,
                 void *r, int64_t ldr, void *z, int64_t ldz, float *stats, void *stream) {
    int rc = check_joint(rows, width, stream_type, type, weight_type, gate_act);
    if (rc) return rc;
    if (rows > 0 && !y && (gate || w_post)) return CP_ERR_ARG;      // (tensors without rows have no address)
    if (!w_pre || (rows > 0 && (!x || !z || (y && !r)))) return CP_ERR_NULL;
    if (rows > 1 && (ldx < width || ldz < width || (y && ldy < width) || (gate && ldg < width) || (r && ldr < width))) return CP_ERR_SIZE;
    const auto of = [&](const void *at, int64_t ld, int t) { return matrix_at(at, rows, width, ld, t); };
    const Extent sums = vector_at(stats, 2 * rows);
    if (in_the_way({of(x, ldx, stream_type), of(y, ldy, type), of(gate, ldg, type)}, {of(r, ldr, stream_type), of(z, ldz, type), sums}, true) ||
        in_the_way({vector_at(w_pre, width, type_bytes(weight_type)), vector_at(w_post, width, type_bytes(weight_type))},
                   {of(r, ldr, stream_type), of(z, ldz, type), sums}))
        return CP_ERR_ARG;
    if (rows == 0) return CP_OK;
    const Joint j{rows, width, x, y, gate, ldx, ldy, ldg, w_pre, w_post, weight_type, gate_act, scale, eps, stats};
    return by_types(stream_type, type, [&](auto ts, auto tb) {
        using TS = decltype(ts);
        using TB = decltype(tb);
        return by_shape<16 / sizeof(TS)>(width, [&](auto nt, auto v, auto nv) {
            constexpr int NT = decltype(nt)::value, V = decltype(v)::value, NV = decltype(nv)::value;
            constexpr int side = Sharing<NT>::kSide;
            const int groups = groups_of(rows, width, 16 / sizeof(TS)) * 2;
            hipLaunchKernelGGL((joint_kernel<TS, TB, NT, V, NV>), dim3((unsigned)std::min<int64_t>((rows + side - 1) / side, groups)), dim3(Sharing<NT>::kThreads), 0,
                               (hipStream_t)stream, j, (TS *)r, ldr, (TB *)z, ldz);
            return launched();
        });
    });
}

int cp_norm_gate_backward_workspace_bytes(int64_t rows, int32_t width, size_t *out_bytes) {
    if (!out_bytes) return CP_ERR_NULL;
    if (rows < 0 || width < 1 || width > CP_NORM_MAX_WIDTH) return CP_ERR_SIZE;
    *out_bytes = 2 * part_bytes(rows, width);
    return CP_OK;
}

int cp_norm_gate_backward(int64_t rows, int32_t width, int stream_type, int type, int weight_type, int gate_act, const void *dr,
                          int64_t lddr, const void *dz, int64_t lddz, const void *x, int64_t ldx, const void *y, int64_t ldy,
                          const void *gate, int64_t ldg, const void *w_pre, const void *w_post, float scale, const float *stats, void *dx,
                          int64_t lddx, void *dy, int64_t lddy, void *dgate, int64_t lddg, void *dw_pre, void *dw_post, void *workspace,
                          size_t workspace_bytes, void *stream) {
    int rc = check_joint(rows, width, stream_type, type, weight_type, gate_act);
    if (rc) return rc;
    if (rows > 0 && !y && (gate || w_post)) return CP_ERR_ARG;
    if (!w_pre || (dw_post && !w_post) || (rows > 0 && dgate && !gate)) return CP_ERR_NULL;
    if (rows > 0 && (!dz || !x || !stats || !dx || (y && !dy))) return CP_ERR_NULL;
    if (rows > 1 && ((dr && lddr < width) || lddz < width || ldx < width || (y && (ldy < width || lddy < width)) || (gate && ldg < width) ||
                     (dgate && lddg < width) || lddx < width))
        return CP_ERR_SIZE;
    const size_t one = part_bytes(rows, width);
    if (dw_pre || dw_post) {
        if (!workspace && rows > 0) return CP_ERR_NULL;
        if ((uintptr_t)workspace % kPolicyAlign || workspace_bytes < 2 * one) return CP_ERR_WORKSPACE;
    }
    const auto of = [&](const void *at, int64_t ld, int t) { return matrix_at(at, rows, width, ld, t); };
    const auto weight = [&](const void *at) { return vector_at(at, width, type_bytes(weight_type)); };
    const Extent e_dr = of(dr, lddr, stream_type), e_dz = of(dz, lddz, type), e_x = of(x, ldx, stream_type), e_y = of(y, ldy, type),
                 e_gate = of(gate, ldg, type), e_dx = of(dx, lddx, stream_type), e_dy = of(dy, lddy, type), e_dgate = of(dgate, lddg, type);
    if (in_the_way({e_dr, e_dz, e_x, e_y, e_gate}, {e_dx, e_dy, e_dgate}, true) ||
        in_the_way({vector_at(stats, 2 * rows), weight(w_pre), weight(w_post)}, {e_dx, e_dy, e_dgate}) ||
        in_the_way({e_dr, e_dz, e_x, e_y, e_gate, vector_at(stats, 2 * rows), e_dx, e_dy, e_dgate}, {weight(dw_pre), weight(dw_post)}))
        return CP_ERR_ARG;
    float *part_pre = dw_pre ? (float *)workspace : nullptr;
    float *part_post = dw_post ? (float *)((char *)workspace + one) : nullptr;
    const Joint j{rows, width, x, y, gate, ldx, ldy, ldg, w_pre, w_post, weight_type, gate_act, scale, 0.0f, (float *)stats};
    const hipStream_t st = (hipStream_t)stream;
    int32_t groups = 0;
    if (rows > 0) {
        rc = by_types(stream_type, type, [&](auto ts, auto tb) {
            using TS = decltype(ts);
            using TB = decltype(tb);
            groups = groups_of(rows, width, 16 / sizeof(TS));
            return by_shape<16 / sizeof(TS)>(width, [&](auto nt, auto v, auto nv) {
                constexpr int NT = decltype(nt)::value, V = decltype(v)::value, NV = decltype(nv)::value;
                const JointGrad<TS, TB> b{(const TS *)dr, (const TB *)dz, (TS *)dx, (TB *)dy, (TB *)dgate, lddr, lddz, lddx, lddy, lddg,
                                          part_pre, part_post};
                constexpr size_t lds = NV * V > 8 ? 2 * NV * V * NT * sizeof(float) : 0;
                auto *kernel = joint_backward_kernel<TS, TB, NT, V, NV>;
                if (lds && hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
                    return (int)CP_ERR_HIP;
                hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(Sharing<NT>::kThreads), lds, st, j, b);
                return launched();
            });
        });
        if (rc) return rc;
    }
    const WeightSum pre{part_pre, dw_pre}, post{part_post, dw_post};
    if (dw_pre || dw_post)
        hipLaunchKernelGGL(weight_sum_kernel, dim3((width + 15) / 16, dw_pre && dw_post ? 2 : 1), dim3(1024), 0, st, dw_pre ? pre : post, post, groups,
                           width, weight_type);
    return launched();
}

}  // extern "C"
