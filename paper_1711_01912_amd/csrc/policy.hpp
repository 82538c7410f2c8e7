// Shared by the operators of a learned placement policy (recurrence.hip, linear_attention.hip, norm_gate.hip, token_logprobs.hip,
// token_sample.hip): element types, vectors of them as they are loaded and stored, and sums over a wavefront.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <initializer_list>
#include <type_traits>

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

// Or past the caches (`stream`): for results of a call that are more than these would keep for the next.  There they only
// displace what is read; 200,000 rows of 1,024 floats, written 16 bytes a lane, took 363 us through the caches and 175 past
// them.
constexpr size_t kStreamed = 64u << 20;      // bytes of results from which on they go past the caches
template <typename T, int V>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, V> &a, bool stream) {
    constexpr int bytes = sizeof(T) * V;
    if constexpr (bytes == 4 || bytes == 8 || bytes == 16) {
        typedef uint32_t word __attribute__((ext_vector_type(bytes / 4)));
        typedef word anywhere __attribute__((aligned(sizeof(T))));
        word w;
        __builtin_memcpy(&w, &a, bytes);
        if (stream) {
            asm volatile("; past");                  // (else the compiler makes one store of both ways, through the caches)
            __builtin_nontemporal_store(w, (anywhere *)p);
            asm volatile("; the caches");
            return;
        }
    }
    store_pack<T, V>(p, a);
}

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
    // the k-th is -inf unless it is to be kept
    __device__ __forceinline__ void set_none(int k, bool keep) {
        if constexpr (sizeof(T) == 4) w[k] = keep ? w[k] : 0xff800000u;
        else {
            const uint32_t none = std::is_same_v<T, bf16> ? 0xff80u : 0xfc00u;
            const uint32_t put = k & 1 ? (w[k / 2] & 0xffffu) | none << 16 : (w[k / 2] & 0xffff0000u) | none;
            w[k / 2] = keep ? w[k / 2] : put;
        }
    }
    // The compiler takes them as new from here on, and in this order.  Without this it converts the rows of a whole run at
    // once, and once for all passes, and spills what it cannot hold.
    __device__ __forceinline__ void renew() {
#pragma unroll
        for (uint32_t &one : w) asm volatile("" : "+v"(one));
    }
};

// sums and maxima over a wavefront's 64 lanes, in every lane
// (by moves inside the vector unit: inside rows of 16 lanes, then from row to row; the last lane has them all)
template <int CTRL, int ROWS>
__device__ __forceinline__ float lane_move(float v, float none) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(none), __float_as_uint(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_sum(float v) {
    v += lane_move<0x111, 0xf>(v, 0.0f);     // row_shr 1, 2, 4, 8
    v += lane_move<0x112, 0xf>(v, 0.0f);
    v += lane_move<0x114, 0xf>(v, 0.0f);
    v += lane_move<0x118, 0xf>(v, 0.0f);
    v += lane_move<0x142, 0xa>(v, 0.0f);     // row_bcast 15, 31
    v += lane_move<0x143, 0xc>(v, 0.0f);
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), kWave - 1));
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}

// one exp and one reciprocal of the hardware (each within an ulp)
__device__ __forceinline__ float fast_exp(float v) { return __builtin_amdgcn_exp2f(v * kLog2e); }
__device__ __forceinline__ float fast_rcp(float v) { return __builtin_amdgcn_rcpf(v); }

// A grid of `groups` workgroups of up to 512 threads, and a workgroup's number in it.  HIP takes fewer than 2^32 threads in a
// dimension; those that the first has no room for go into the second, whose last row may have some too many.
constexpr uint32_t kGridX = 1u << 22;
inline dim3 grid_of(int64_t groups) {
    return dim3((unsigned)(groups < kGridX ? groups : kGridX), (unsigned)((groups + kGridX - 1) / kGridX));
}
__device__ __forceinline__ uint32_t group_number() { return blockIdx.y * kGridX + blockIdx.x; }

inline size_t type_bytes(int type) { return type == CP_TYPE_F32 ? 4 : 2; }
inline bool known_type(int type) { return type == CP_TYPE_F32 || type == CP_TYPE_BF16 || type == CP_TYPE_F16; }
inline size_t align_up(size_t v) { return (v + kPolicyAlign - 1) / kPolicyAlign * kPolicyAlign; }
inline int launched() { return hipGetLastError() == hipSuccess ? CP_OK : CP_ERR_HIP; }

// An array of rows in memory (of a vector: one row), for whether a result lies where something else does.  at: null, if there is
// none
struct Extent {
    const void *at;
    int64_t rows, bytes, pitch;          // of a row; from a row to the next
    size_t each;                         // of an element
};
inline Extent matrix_at(const void *at, int64_t rows, int32_t width, int64_t ld, int type) {
    const int64_t each = (int64_t)type_bytes(type);
    return {at, rows, width * each, (rows > 1 ? ld : width) * each, (size_t)each};
}
inline Extent vector_at(const void *at, int64_t count, size_t each = sizeof(float)) { return {at, 1, count * (int64_t)each, count * (int64_t)each, each}; }

// whether they share any byte (the rows of two slices of one buffer lie between each other and share none)
inline bool share(const Extent &a, const Extent &b) {
    if (!a.at || !b.at || a.rows < 1 || b.rows < 1 || a.bytes < 1 || b.bytes < 1) return false;
    const int64_t pa = (int64_t)(uintptr_t)a.at, pb = (int64_t)(uintptr_t)b.at;
    if (pa + (a.rows - 1) * a.pitch + a.bytes <= pb || pb + (b.rows - 1) * b.pitch + b.bytes <= pa) return false;
    const int64_t pitch = a.rows > 1 ? a.pitch : b.pitch;
    if ((a.rows == 1 && b.rows == 1) || pitch < a.bytes || pitch < b.bytes || (a.rows > 1 && b.rows > 1 && a.pitch != b.pitch)) return true;
    // b's first row begins `off` bytes behind the start of a's row number `row`, if a had rows without end both ways
    int64_t row = (pb - pa) / pitch, off = (pb - pa) % pitch;
    if (off < 0) row--, off += pitch;
    auto meet = [&](int64_t first) { return first < a.rows && first + b.rows > 0; };
    return (off < a.bytes && meet(row)) || (off + b.bytes > pitch && meet(row + 1));
}
// whether they are one and the same, element upon element
inline bool same(const Extent &a, const Extent &b) {
    return a.at == b.at && a.rows == b.rows && a.bytes == b.bytes && a.pitch == b.pitch && a.each == b.each;
}

// Whether a result shares memory with another result or with an input; `in_place`: it may be one of the inputs
inline bool in_the_way(std::initializer_list<Extent> in, std::initializer_list<Extent> out, bool in_place = false) {
    for (const Extent *o = out.begin(); o != out.end(); o++) {
        for (const Extent &i : in)
            if (share(i, *o) && !(in_place && same(i, *o))) return true;
        for (const Extent *p = out.begin(); p != o; p++)
            if (share(*p, *o)) return true;
    }
    return false;
}

// calls f with a value of the element type that `type` names
template <typename F>
inline auto by_type(int type, F f) {
    if (type == CP_TYPE_F32) return f(float{});
    if (type == CP_TYPE_BF16) return f(bf16{});
    return f(f16{});
}

}  // namespace cpeval
