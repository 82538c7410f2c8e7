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
// Bound by memory: a row is held in registers by one workgroup, so that every input is read once and every output written
// once.  Sums are floats; a result is rounded once, to its type.
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

__device__ __forceinline__ float weight(const void *w, int type, int64_t c) {
    if (type == CP_TYPE_F32) return ((const float *)w)[c];
    return type == CP_TYPE_BF16 ? (float)((const bf16 *)w)[c] : (float)((const f16 *)w)[c];
}

// sum over a workgroup, in every thread
template <int NT>
__device__ __forceinline__ float group_sum(float v, float *lds) {
    v = wave_sum(v);
    if (NT == kWave) return v;
    const int wave = threadIdx.x / kWave;
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) lds[wave] = v;
    __syncthreads();
    float all = 0.0f;
#pragma unroll
    for (int w = 0; w < NT / kWave; w++) all += lds[w];
    return all;
}

// act(gate) and its slope
__device__ __forceinline__ void gate_of(float g, int act, float &value, float &slope) {
    const float sg = fast_rcp(1.0f + fast_exp(-g));
    if (act == CP_GATE_SIGMOID) {
        value = sg;
        slope = sg * (1.0f - sg);
    } else if (act == CP_GATE_SILU) {
        value = g * sg;
        slope = sg * (1.0f + g * (1.0f - sg));
    } else {
        value = g;
        slope = 1.0f;
    }
}

// TS: the stream's type (x, r, dx, dr), TB: the block's (y, gate, z and their gradients)
template <typename TS, typename TB, int NT, int V, int NV>
__global__ __launch_bounds__(NT) void joint_kernel(Joint j, TS *r_out, int64_t ldr, TB *z_out, int64_t ldz) {
    __shared__ float lds[NT / kWave];
    const float inv = 1.0f / j.width;
    for (int64_t row = blockIdx.x; row < j.rows; row += gridDim.x) {
        Pack<TS, V> x[NV];
        Pack<TB, V> y[NV], g[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int64_t c = ((int64_t)i * NT + threadIdx.x) * V;
            if (c >= j.width) continue;
            x[i] = load_pack<TS, V>((const TS *)j.x + row * j.ldx + c);
            if (j.y) y[i] = load_pack<TB, V>((const TB *)j.y + row * j.ldy + c);
            if (j.gate) g[i] = load_pack<TB, V>((const TB *)j.gate + row * j.ldg + c);
        }
        float ry = 1.0f;
        if (j.y && j.w_post) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; i++) {
                if (((int64_t)i * NT + threadIdx.x) * V >= j.width) continue;
#pragma unroll
                for (int k = 0; k < V; k++) sum = fmaf((float)y[i].v[k], (float)y[i].v[k], sum);
            }
            ry = 1.0f / sqrtf(group_sum<NT>(sum, lds) * inv + j.eps);
        }
        float r[NV][V], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int64_t c = ((int64_t)i * NT + threadIdx.x) * V;
            if (c >= j.width) continue;
            Pack<TS, V> out;
#pragma unroll
            for (int k = 0; k < V; k++) {
                r[i][k] = (float)x[i].v[k];
                if (j.y) {
                    float value = 1.0f, slope, u = (float)y[i].v[k];
                    if (j.gate) gate_of((float)g[i].v[k], j.act, value, slope);
                    if (j.w_post) u = u * ry * weight(j.w_post, j.weight_type, c + k);
                    r[i][k] = fmaf(j.scale * value, u, r[i][k]);
                }
                out.v[k] = (TS)r[i][k];
                sum = fmaf(r[i][k], r[i][k], sum);
            }
            if (r_out) store_pack<TS, V>(r_out + row * ldr + c, out);
        }
        const float rr = 1.0f / sqrtf(group_sum<NT>(sum, lds) * inv + j.eps);
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int64_t c = ((int64_t)i * NT + threadIdx.x) * V;
            if (c >= j.width) continue;
            Pack<TB, V> out;
#pragma unroll
            for (int k = 0; k < V; k++) out.v[k] = (TB)(r[i][k] * rr * weight(j.w_pre, j.weight_type, c + k));
            store_pack<TB, V>(z_out + row * ldz + c, out);
        }
        if (j.stats && threadIdx.x == 0) {
            j.stats[row] = ry;
            j.stats[j.rows + row] = rr;
        }
    }
}

template <typename TS, typename TB, int NT, int V, int NV>
__global__ __launch_bounds__(NT) void joint_backward_kernel(Joint j, const TS *dr, int64_t lddr, const TB *dz, int64_t lddz, TS *dx,
                                                            int64_t lddx, TB *dy, int64_t lddy, TB *dg, int64_t lddg, float *part_pre,
                                                            float *part_post) {
    __shared__ float lds[NT / kWave];
    const float inv = 1.0f / j.width;
    float acc_pre[NV][V], acc_post[NV][V];
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
        for (int k = 0; k < V; k++) acc_pre[i][k] = acc_post[i][k] = 0.0f;
    for (int64_t row = blockIdx.x; row < j.rows; row += gridDim.x) {
        const float ry = j.w_post ? j.stats[row] : 1.0f, rr = j.stats[j.rows + row];
        Pack<TS, V> x[NV], d[NV];
        Pack<TB, V> y[NV], g[NV], e[NV];
        float rh[NV][V], dot = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int64_t c = ((int64_t)i * NT + threadIdx.x) * V;
            if (c >= j.width) continue;
            x[i] = load_pack<TS, V>((const TS *)j.x + row * j.ldx + c);
            if (j.y) y[i] = load_pack<TB, V>((const TB *)j.y + row * j.ldy + c);
            if (j.gate) g[i] = load_pack<TB, V>((const TB *)j.gate + row * j.ldg + c);
            if (dr) d[i] = load_pack<TS, V>(dr + row * lddr + c);
            e[i] = load_pack<TB, V>(dz + row * lddz + c);
        }
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int64_t c = ((int64_t)i * NT + threadIdx.x) * V;
            if (c >= j.width) continue;
#pragma unroll
            for (int k = 0; k < V; k++) {
                float r = (float)x[i].v[k];
                if (j.y) {
                    float value = 1.0f, slope, u = (float)y[i].v[k];
                    if (j.gate) gate_of((float)g[i].v[k], j.act, value, slope);
                    if (j.w_post) u = u * ry * weight(j.w_post, j.weight_type, c + k);
                    r = fmaf(j.scale * value, u, r);
                }
                rh[i][k] = r * rr;
                const float dzv = (float)e[i].v[k];
                acc_pre[i][k] = fmaf(dzv, rh[i][k], acc_pre[i][k]);
                dot = fmaf(dzv * weight(j.w_pre, j.weight_type, c + k), rh[i][k], dot);
            }
        }
        dot = group_sum<NT>(dot, lds) * inv;
        float du[NV][V], dot2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int64_t c = ((int64_t)i * NT + threadIdx.x) * V;
            if (c >= j.width) continue;
            Pack<TS, V> ox;
            Pack<TB, V> og;
#pragma unroll
            for (int k = 0; k < V; k++) {
                float q = rr * ((float)e[i].v[k] * weight(j.w_pre, j.weight_type, c + k) - rh[i][k] * dot);
                if (dr) q += (float)d[i].v[k];
                ox.v[k] = (TS)q;
                if (j.y) {
                    float value = 1.0f, slope = 0.0f, yh = (float)y[i].v[k], w = 1.0f;
                    if (j.gate) gate_of((float)g[i].v[k], j.act, value, slope);
                    if (j.w_post) {
                        yh *= ry;
                        w = weight(j.w_post, j.weight_type, c + k);
                    }
                    const float qs = q * j.scale;
                    og.v[k] = (TB)(qs * yh * w * slope);
                    const float dv = qs * value;
                    acc_post[i][k] = fmaf(dv, yh, acc_post[i][k]);
                    du[i][k] = dv * w;
                    dot2 = fmaf(du[i][k], yh, dot2);
                }
            }
            store_pack<TS, V>(dx + row * lddx + c, ox);
            if (dg) store_pack<TB, V>(dg + row * lddg + c, og);
        }
        if (!j.y) continue;
        if (j.w_post) dot2 = group_sum<NT>(dot2, lds) * inv;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int64_t c = ((int64_t)i * NT + threadIdx.x) * V;
            if (c >= j.width) continue;
            Pack<TB, V> oy;
#pragma unroll
            for (int k = 0; k < V; k++) oy.v[k] = (TB)(j.w_post ? ry * (du[i][k] - (float)y[i].v[k] * ry * dot2) : du[i][k]);
            store_pack<TB, V>(dy + row * lddy + c, oy);
        }
    }
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int64_t c = ((int64_t)i * NT + threadIdx.x) * V;
        if (c >= j.width) continue;
#pragma unroll
        for (int k = 0; k < V; k++) {
            if (part_pre) part_pre[(int64_t)blockIdx.x * j.width + c + k] = acc_pre[i][k];
            if (part_post) part_post[(int64_t)blockIdx.x * j.width + c + k] = acc_post[i][k];
        }
    }
}

// a weight's gradient from the workgroups' sums, in a fixed order and in 64 bits
__global__ __launch_bounds__(256) void weight_sum_kernel(const float *part, int32_t groups, int32_t width, void *out, int type) {
    __shared__ double lds[4][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t c = (int64_t)blockIdx.x * kWave + lane;
    double sum = 0.0;
    if (c < width)
        for (int32_t i = wave; i < groups; i += 4) sum += part[(int64_t)i * width + c];
    lds[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || c >= width) return;
    const float all = (float)(((lds[0][lane] + lds[1][lane]) + lds[2][lane]) + lds[3][lane]);
    if (type == CP_TYPE_F32) ((float *)out)[c] = all;
    else if (type == CP_TYPE_BF16) ((bf16 *)out)[c] = (bf16)all;
    else ((f16 *)out)[c] = (f16)all;
}

constexpr int32_t kMostGroups = 2048;

// calls f(threads, values a load, loads a thread) for the smallest workgroup that holds a row
template <typename F>
int by_shape(bool wide, int32_t width, F f) {
    auto of = [&](auto v) {
        constexpr int V = decltype(v)::value;
        auto go = [&](auto nt, auto nv) { return f(nt, v, nv); };
        using std::integral_constant;
        if (width <= 64 * V) return go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
        if (width <= 256 * V) return go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
        if (width <= 512 * V) return go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
        if (width <= 1024 * V) return go(integral_constant<int, 512>{}, integral_constant<int, 2>{});
        if (width <= 2048 * V) return go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
        if (width <= 4096 * V) return go(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
        if (V == 1 && width <= 8192) return go(integral_constant<int, 1024>{}, integral_constant<int, V == 1 ? 8 : 4>{});
        if (V == 1 && width <= 16384) return go(integral_constant<int, 1024>{}, integral_constant<int, V == 1 ? 16 : 4>{});
        return (int)CP_ERR_SIZE;
    };
    if (wide) return of(std::integral_constant<int, 4>{});
    return of(std::integral_constant<int, 1>{});
}

int check_joint(int64_t rows, int32_t width, int stream_type, int type, int weight_type, int act) {
    if (!known_type(stream_type) || !known_type(type) || !known_type(weight_type)) return CP_ERR_ARG;
    if ((stream_type != type && stream_type != CP_TYPE_F32) || act < CP_GATE_NONE || act > CP_GATE_SILU) return CP_ERR_ARG;
    if (rows < 0 || width < 1 || width > CP_NORM_MAX_WIDTH) return CP_ERR_SIZE;
    return CP_OK;
}

bool aligned(size_t bytes, std::initializer_list<const void *> at, std::initializer_list<int64_t> ld) {
    for (const void *p : at)
        if ((uintptr_t)p % (4 * bytes)) return false;
    for (int64_t d : ld)
        if (d % 4) return false;
    return true;
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
    if (rows == 0) return CP_OK;
    const Joint j{rows, width, x, y, gate, ldx, y ? ldy : 0, gate ? ldg : 0, w_pre, w_post, weight_type, gate_act, scale, eps, stats};
    const bool wide = width % 4 == 0 && aligned(type_bytes(stream_type), {x, r}, {ldx, r ? ldr : 0}) &&
                      aligned(type_bytes(type), {y, gate, z}, {j.ldy, j.ldg, ldz});
    return by_types(stream_type, type, [&](auto ts, auto tb) {
        using TS = decltype(ts);
        using TB = decltype(tb);
        return by_shape(wide, width, [&](auto nt, auto v, auto nv) {
            constexpr int NT = decltype(nt)::value, V = decltype(v)::value, NV = decltype(nv)::value;
            hipLaunchKernelGGL((joint_kernel<TS, TB, NT, V, NV>), dim3((unsigned)std::min<int64_t>(rows, 256 * 64)), dim3(NT), 0,
                               (hipStream_t)stream, j, (TS *)r, ldr, (TB *)z, ldz);
            return launched();
        });
    });
}

int cp_norm_gate_backward_workspace_bytes(int64_t rows, int32_t width, size_t *out_bytes) {
    if (!out_bytes) return CP_ERR_NULL;
    if (rows < 0 || width < 1 || width > CP_NORM_MAX_WIDTH) return CP_ERR_SIZE;
    *out_bytes = 2 * align_up((size_t)std::min<int64_t>(rows, kMostGroups) * width * sizeof(float));
    return CP_OK;
}

int cp_norm_gate_backward(int64_t rows, int32_t width, int stream_type, int type, int weight_type, int gate_act, const void *dr,
                          int64_t lddr, const void *dz, int64_t lddz, const void *x, int64_t ldx, const void *y, int64_t ldy,
                          const void *gate, int64_t ldg, const void *w_pre, const void *w_post, float scale, const float *stats, void *dx,
                          int64_t lddx, void *dy, int64_t lddy, void *dgate, int64_t lddg, void *dw_pre, void *dw_post, void *workspace,
                          size_t workspace_bytes, void *stream) {
    int rc = check_joint(rows, width, stream_type, type, weight_type, gate_act);
    if (rc) return rc;
    if (rows > 0 && !y && (gate || w_post)) return CP_ERR_ARG;      // (tensors without rows have no address)
    if (!w_pre || (dw_post && !w_post) || (rows > 0 && dgate && !gate)) return CP_ERR_NULL;
    if (rows > 0 && (!dz || !x || !stats || !dx || (y && !dy))) return CP_ERR_NULL;
    if (rows > 1 && ((dr && lddr < width) || lddz < width || ldx < width || (y && (ldy < width || lddy < width)) || (gate && ldg < width) ||
                     (dgate && lddg < width) || lddx < width))
        return CP_ERR_SIZE;
    const int32_t groups = (int32_t)std::min<int64_t>(rows, kMostGroups);
    const size_t one = align_up((size_t)groups * width * sizeof(float));
    if (dw_pre || dw_post) {
        if (!workspace && rows > 0) return CP_ERR_NULL;
        if ((uintptr_t)workspace % kPolicyAlign || workspace_bytes < 2 * one) return CP_ERR_WORKSPACE;
    }
    float *part_pre = dw_pre ? (float *)workspace : nullptr;
    float *part_post = dw_post ? (float *)((char *)workspace + one) : nullptr;
    const Joint j{rows, width, x, y, gate, ldx, y ? ldy : 0, gate ? ldg : 0, w_pre, w_post, weight_type, gate_act, scale, 0.0f, (float *)stats};
    const bool wide = width % 4 == 0 && aligned(type_bytes(stream_type), {x, dx, dr}, {ldx, lddx, dr ? lddr : 0}) &&
                      aligned(type_bytes(type), {y, gate, dz, y ? dy : nullptr, dgate}, {j.ldy, j.ldg, lddz, y ? lddy : 0, dgate ? lddg : 0});
    const hipStream_t st = (hipStream_t)stream;
    if (rows > 0) {
        rc = by_types(stream_type, type, [&](auto ts, auto tb) {
            using TS = decltype(ts);
            using TB = decltype(tb);
            return by_shape(wide, width, [&](auto nt, auto v, auto nv) {
                constexpr int NT = decltype(nt)::value, V = decltype(v)::value, NV = decltype(nv)::value;
                hipLaunchKernelGGL((joint_backward_kernel<TS, TB, NT, V, NV>), dim3((unsigned)groups), dim3(NT), 0, st, j, (const TS *)dr, lddr,
                                   (const TB *)dz, lddz, (TS *)dx, lddx, (TB *)dy, lddy, (TB *)dgate, lddg, part_pre, part_post);
                return launched();
            });
        });
        if (rc) return rc;
    }
    if (dw_pre)
        hipLaunchKernelGGL(weight_sum_kernel, dim3((width + kWave - 1) / kWave), dim3(256), 0, st, part_pre, groups, width, dw_pre, weight_type);
    if (dw_post)
        hipLaunchKernelGGL(weight_sum_kernel, dim3((width + kWave - 1) / kWave), dim3(256), 0, st, part_post, groups, width, dw_post, weight_type);
    return launched();
}

}  // extern "C"
