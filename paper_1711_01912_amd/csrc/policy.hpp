// Shared by the operators of a learned placement policy (recurrence.hip, norm_gate.hip, token_logprobs.hip): element types,
// vectors of them as they are loaded and stored, and sums over a wavefront.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/cpeval.h"

namespace cpeval {

constexpr int kWave = 64;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr size_t kPolicyAlign = 256;     // of workspaces, as cp_eval's

using bf16 = __bf16;
using f16 = _Float16;

// V values as one load or store, wherever a value may lie: global memory takes wide accesses at any element's address, and
// rows of odd widths and distances are read as those of even ones
template <typename T, int V>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
    T v[V];
};

template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T *p) {
    return *reinterpret_cast<const Pack<T, V> *>(p);
}

template <typename T, int V>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, V> &a) {
    *reinterpret_cast<Pack<T, V> *>(p) = a;
}

// sums and maxima over a wavefront's 64 lanes, in every lane
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}

// one exp and one reciprocal of the hardware (each within an ulp)
__device__ __forceinline__ float fast_exp(float v) { return __builtin_amdgcn_exp2f(v * kLog2e); }
__device__ __forceinline__ float fast_rcp(float v) { return __builtin_amdgcn_rcpf(v); }

inline size_t type_bytes(int type) { return type == CP_TYPE_F32 ? 4 : 2; }
inline bool known_type(int type) { return type == CP_TYPE_F32 || type == CP_TYPE_BF16 || type == CP_TYPE_F16; }
inline size_t align_up(size_t v) { return (v + kPolicyAlign - 1) / kPolicyAlign * kPolicyAlign; }
inline int launched() { return hipGetLastError() == hipSuccess ? CP_OK : CP_ERR_HIP; }

// calls f with a value of the element type that `type` names
template <typename F>
inline auto by_type(int type, F f) {
    if (type == CP_TYPE_F32) return f(float{});
    if (type == CP_TYPE_BF16) return f(bf16{});
    return f(f16{});
}

}  // namespace cpeval
