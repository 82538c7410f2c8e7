// What the kernels of cp_linear_attention share: the pass over rows with a matrix a head as its state, its operands, the cutting
// of rows into segments, sequences and chunks, and the fragments that the matrix instructions take.
#pragma once

#include <climits>

#include "policy.hpp"

namespace cpeval {
namespace attention {

constexpr int kThreads = 256;            // of the kernels beside the pass

// rows [rows][heads][width]: element c of head h of row r at r * ld + (h / group) * hd + c
struct Operand {
    const void *at;
    int64_t ld, hd;
    int32_t group = 1;                   // (heads are divided by it, also of an operand that a pass does not have)
};

// One pass: S_t = gamma S_{t-1} + s_in b_t^T x_t and o_t = s_out a_t S_t along the rows of each sequence, S of wa x wb.  The forward call
// is one (a, b, x = q, k, v), dq one with (do, v, k), and, from the last row on, dv one with (k, q, do) and dk with (v, do, q).
// There the state is the gradient of S: it takes part in its own row undecayed (shift 1: gamma^0 for the first row after it).
struct Pass {
    int64_t rows, len;                   // len: of a sequence, without ptr
    const int32_t *ptr;                  // [num_seq + 1], or null
    int32_t num_seq, segments, parts;    // parts: segments of a sequence, without ptr
    int64_t seg_rows;
    int32_t heads, wa, wb, slices;       // slices: workgroups side by side along wb
    bool back, transposed;               // back: from the last row to the first; transposed: states lie in memory as [wb][wa]
    int32_t shift;
    float s_in, s_out;
    const float *log_decay;
    Operand a, b, x;
    const float *init;                   // [num_seq][heads][..] or null
    const float *enter;                  // [segments][heads][..], states that enter segments, or null (no sequence is cut)
    float *last;                         // [num_seq][heads][..] or null
    void *o;                             // rows as a's heads
    int64_t ldo, hdo;
    bool wide;                           // o in floats, whatever the type
    bool last_first;                     // chunks as those of a pass from the other end
    // of passes that add to the decays' gradient
    Operand d;                           // what o is the gradient of
    const float *dlast, *denter;         // gradients of the states behind sequences and segments, or null
    double *part;                        // of a head: [segments][slices], part_step from head to head
    int64_t part_step;
};

// ---- sequences ---------------------------------------------------------------------------------------

// rows [lo, hi) of a segment
__device__ __forceinline__ void segment_of(const Pass &p, int32_t s, int64_t &lo, int64_t &hi) {
    if (p.ptr) {
        const int64_t total = min((int64_t)max(p.ptr[p.num_seq], 0), p.rows);
        lo = min(s * p.seg_rows, total), hi = min(lo + p.seg_rows, total);
    } else {
        const int64_t seq = s / p.parts, from = seq * p.len;
        lo = from + (s % p.parts) * p.seg_rows, hi = min(lo + p.seg_rows, from + p.len);
    }
}

// The rows of one sequence inside a segment, in the order of the pass.  (Whatever ptr holds, pieces lie inside the segment and
// hold a row at least.)
struct Piece {
    int64_t lo, hi;
    int32_t seq;
    bool starts, ends;                   // whether the sequence does, in the order of the pass
};

__device__ __forceinline__ Piece piece_at(const Pass &p, int64_t lo, int64_t hi) {
    const int64_t row = p.back ? hi - 1 : lo;
    Piece a;
    int64_t from, to;
    if (p.ptr) {
        int32_t l = 0, r = p.num_seq;    // the last sequence that begins at or before the row
        while (r - l > 1) {
            const int32_t m = l + (r - l) / 2;
            if (p.ptr[m] <= row) l = m;
            else r = m;
        }
        a.seq = l;
        from = p.ptr[l], to = p.ptr[l + 1];
    } else {
        a.seq = (int32_t)(row / p.len);
        from = a.seq * p.len, to = from + p.len;
    }
    if (p.back) {
        a.hi = hi, a.lo = max(lo, min(from, hi - 1));
        a.starts = to <= hi, a.ends = from >= lo;
    } else {
        a.lo = lo, a.hi = min(hi, max(to, lo + 1));
        a.starts = from >= lo, a.ends = to <= hi;
    }
    return a;
}

// ---- decays ------------------------------------------------------------------------------------------

// A head's decay: its logarithm, and that to base 2 in two parts.  (An error of it is the same in every row: over a million
// rows of four heads, the slowest with a decay of 6e-4 a row, the decays' gradient was off by 6.7e-8 with the first part alone and is by 1.2e-8
// with both.  Heads of 2.5e-4 stay at 2e-7 to 6e-7, the roundings of states in 32 bits.)  So far below one that any power is 0, it is as good as
// that: 0 * inf does not come up.  Above 0, or NaN: NaN.
struct Decay {
    float log, hi, lo;
};
__device__ __forceinline__ Decay decay_of(float log_decay) {
    constexpr float kLog2eLow = (float)(1.44269504088896340736 - (double)kLog2e);
    Decay d;
    d.log = log_decay <= 0.0f ? fmaxf(log_decay, -700.0f) : __uint_as_float(0x7fc00000u);
    d.hi = d.log * kLog2e;
    d.lo = fmaf(d.log, kLog2e, -d.hi) + d.log * kLog2eLow;
    return d;
}
__device__ __forceinline__ float power(const Decay &d, int n) {
    const float by = (float)n, hi = d.hi * by, lo = fmaf(d.lo, by, fmaf(d.hi, by, -hi)), e = __builtin_amdgcn_exp2f(hi);
    return fmaf(e, lo * kLn2, e);
}
// gamma^n - 1: states are decayed as S + S (gamma^n - 1), which is off by half a step of S where the rounding of a gamma^n close to one
// would add up along a head's whole memory
__device__ __forceinline__ float power_less_one(const Decay &d, int n) { return expm1f(d.log * (float)n); }

// A state times gamma^n: of a decay above a half as S + S (gamma^n - 1), see above; of one below, where that difference would lose what it
// has fewer bits than, by gamma^n itself
struct Fade {
    float by;
    bool near;
};
__device__ __forceinline__ Fade fade_of(const Decay &d, int n) {
    const float less = power_less_one(d, n);
    return less >= -0.5f ? Fade{less, true} : Fade{power(d, n), false};
}
__device__ __forceinline__ float faded(float s, const Fade &f) { return fmaf(s, f.by, f.near ? s : 0.0f); }

// What a segment does to the state before it
struct Gain {
    Fade fade;
    bool drops;                          // none of it is left: a sequence began
};

// ---- fragments ---------------------------------------------------------------------------------------

typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Elements as the matrix instructions take them.  bf16 as it is; fp16 as the sum of two bf16, which is exact; what is computed in 32
// bits (states, scores, decayed rows) as the sum of three bf16, which is exact too: two would be off by up to 2^-16, and round one output of bf16
// in 230 and of fp16 in 28 to the wrong side of a middle; with three it is one in 4,500 and in 700.  float as it is, through the float
// instructions.
template <typename T>
struct Form {
    using E = bf16;
    static constexpr int kPlanes = 1, kSplit = 3;
};
template <>
struct Form<f16> {
    using E = bf16;
    static constexpr int kPlanes = 2, kSplit = 3;
};
template <>
struct Form<float> {
    using E = float;
    static constexpr int kPlanes = 1, kSplit = 1;
};

// 16 x 32 of a matrix in a wavefront: lane l holds, of row (or column) l % 16, places 4 (l / 16) + 0..3 and 16 + 4 (l / 16) + 0..3.
// That is a result tile's own layout (4 of 16 rows a lane, two tiles), so that states and scores go from results to operands where they are;
// the order of places in a product does not matter as long as both operands have the same.
template <typename E, int P>
struct Frag {
    bf16x8 p[P];
};
template <>
struct Frag<float, 1> {
    float v[8];
};

// (the smallest parts first; parts that together lie beyond the finer operand's last are left out, unless all are asked for)
template <bool ALL = false, int PA, int PB>
__device__ __forceinline__ f32x4 product(const Frag<bf16, PA> &a, const Frag<bf16, PB> &b, f32x4 c) {
    constexpr int kMost = ALL ? PA + PB - 1 : PA > PB ? PA : PB;
#pragma unroll
    for (int s = kMost - 1; s >= 0; s--)
#pragma unroll
        for (int i = 0; i < PA; i++) {
            const int j = s - i;
            if (j >= 0 && j < PB) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[j], c, 0, 0, 0);
        }
    return c;
}
template <bool ALL = false>
__device__ __forceinline__ f32x4 product(const Frag<float, 1> &a, const Frag<float, 1> &b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 8; i++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], c, 0, 0, 0);
    return c;
}

// N results at once, part by part, so that neighbouring instructions do not wait for each other: c[k] += a[k] b, or b a[k] if TURNED
template <bool TURNED = false, int N, int PA, int PB>
__device__ __forceinline__ void products(const Frag<bf16, PA> (&a)[N], const Frag<bf16, PB> &b, f32x4 *c) {
    constexpr int kMost = PA > PB ? PA : PB;
#pragma unroll
    for (int s = kMost - 1; s >= 0; s--)
#pragma unroll
        for (int i = 0; i < PA; i++) {
            const int j = s - i;
            if (j >= 0 && j < PB) {
#pragma unroll
                for (int k = 0; k < N; k++)
                    c[k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(TURNED ? b.p[j] : a[k].p[i], TURNED ? a[k].p[i] : b.p[j], c[k], 0, 0, 0);
            }
        }
}
template <bool TURNED = false, int N>
__device__ __forceinline__ void products(const Frag<float, 1> (&a)[N], const Frag<float, 1> &b, f32x4 *c) {
#pragma unroll
    for (int i = 0; i < 8; i++)
#pragma unroll
        for (int k = 0; k < N; k++) c[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(TURNED ? b.v[i] : a[k].v[i], TURNED ? a[k].v[i] : b.v[i], c[k], 0, 0, 0);
}
// What was asked of LDS before it is under way before what comes after it begins.  (The compiler else asks for each operand right
// before its product and waits for it.)
__device__ __forceinline__ void asked() { __builtin_amdgcn_sched_barrier(0); }

__device__ __forceinline__ void split(const float (&v)[8], Frag<float, 1> &f) {
#pragma unroll
    for (int e = 0; e < 8; e++) f.v[e] = v[e];
}
// The parts of two values, each part's in one word: all but the last are the upper half of what is left, the last is rounded.  (Three hold all
// 24 bits of a float.)
template <int P>
__device__ __forceinline__ void parts(float a, float b, uint32_t (&w)[P]) {
#pragma unroll
    for (int i = 0; i + 1 < P; i++) {
        w[i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
        a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
        b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
    }
    typedef bf16 pair __attribute__((ext_vector_type(2)));
    w[P - 1] = __builtin_bit_cast(uint32_t, pair{(bf16)a, (bf16)b});
}
template <int P>
__device__ __forceinline__ void split(const float (&v)[8], Frag<bf16, P> &f) {
    uint32_t w[P][4];
#pragma unroll
    for (int e = 0; e < 4; e++) {
        uint32_t two[P];
        parts<P>(v[2 * e], v[2 * e + 1], two);
#pragma unroll
        for (int i = 0; i < P; i++) w[i][e] = two[i];
    }
#pragma unroll
    for (int i = 0; i < P; i++) __builtin_memcpy(&f.p[i], w[i], sizeof(w[i]));
}
template <typename E, int P>
__device__ __forceinline__ void split(f32x4 a, f32x4 b, Frag<E, P> &f) {
    const float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    split(v, f);
}
__device__ __forceinline__ void values(const Frag<float, 1> &f, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = f.v[e];
}
template <int P>
__device__ __forceinline__ void values(const Frag<bf16, P> &f, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
        v[e] = (float)f.p[0][e];
        if constexpr (P > 1) v[e] += (float)f.p[1][e];
    }
}

// R rows of a chunk in LDS, 32 bytes more from row to row than they hold: then the lanes of an instruction meet in no bank, whether they read
// 16 bytes along rows (4.4 cycles; 8.4 with 16 bytes more) or across them (2.8 cycles; 4.8).
// ORDERED: of 32 places those that a lane reads along a row, 4 and 4 that are 16 apart, are neighbours.
template <typename E, int P, int W, int R, bool ORDERED>
struct Tile {
    static constexpr int kPitch = W + 32 / (int)sizeof(E);
    static constexpr bool kOrdered = ORDERED && sizeof(E) == 2;
    E at[P][R][kPitch];

    // where 4 places from c on lie
    __device__ __forceinline__ static int place(int c) { return kOrdered ? c / 32 * 32 + c % 16 * 2 + c % 32 / 16 * 4 : c; }

    // rows r0 + 0..15, places 32 kb + 0..31
    __device__ __forceinline__ Frag<E, P> along(int r0, int kb, int lane) const {
        Frag<E, P> f;
        const int row = r0 + lane % 16, c = 32 * kb + 4 * (lane / 16);
        if constexpr (sizeof(E) == 4) {
            const f32x4 a = *(const f32x4 *)&at[0][row][c], b = *(const f32x4 *)&at[0][row][c + 16];
#pragma unroll
            for (int e = 0; e < 4; e++) f.v[e] = a[e], f.v[4 + e] = b[e];
        } else {
#pragma unroll
            for (int i = 0; i < P; i++) {
                if constexpr (kOrdered) f.p[i] = *(const bf16x8 *)&at[i][row][place(c)];
                else {
                    const bf16x4 a = *(const bf16x4 *)&at[i][row][c], b = *(const bf16x4 *)&at[i][row][c + 16];
                    f.p[i] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
                }
            }
        }
        return f;
    }
    // columns c0 + 0..15, rows 32 jb + 0..31 as places (16 bits: transposed as they are read, 4 rows of 16 places by 16 lanes)
    __device__ __forceinline__ Frag<E, P> across(int c0, int jb, int lane) const {
        static_assert(!kOrdered);
        Frag<E, P> f;
        const int i = lane % 16, row = 32 * jb + 4 * (lane / 16);
        if constexpr (sizeof(E) == 4) {
#pragma unroll
            for (int e = 0; e < 4; e++) f.v[e] = at[0][row + e][c0 + i], f.v[4 + e] = at[0][row + 16 + e][c0 + i];
        } else {
            typedef __attribute__((address_space(3))) bf16x4 *Lds;
#pragma unroll
            for (int k = 0; k < P; k++) {
                const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((Lds)&at[k][row + i / 4][c0 + 4 * (i % 4)]);
                const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((Lds)&at[k][row + 16 + i / 4][c0 + 4 * (i % 4)]);
                f.p[k] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
            }
        }
        return f;
    }
    // 8 places from c on, a multiple of 8, of a row
    __device__ __forceinline__ void put(int plane, int row, int c, const Pack<E, 8> &v) {
        if constexpr (kOrdered) {
            bf16x4 half[2];
            __builtin_memcpy(half, &v, sizeof(half));
            *(bf16x4 *)&at[plane][row][place(c)] = half[0];
            *(bf16x4 *)&at[plane][row][place(c) + 8] = half[1];
        } else *(Pack<E, 8> *)__builtin_assume_aligned(&at[plane][row][c], 16) = v;
    }
    // 4 places from c on of a row, as what is computed is kept
    __device__ __forceinline__ void keep(int row, int c, f32x4 v) {
        if constexpr (sizeof(E) == 4) *(f32x4 *)&at[0][row][c] = v;
        else {
            uint32_t one[P], two[P];
            parts<P>(v[0], v[1], one);
            parts<P>(v[2], v[3], two);
#pragma unroll
            for (int i = 0; i < P; i++) *(uint2 *)&at[i][row][place(c)] = uint2{one[i], two[i]};
        }
    }
};

// whether 8 values hold an infinity or a NaN: all ones in an exponent
template <typename T>
__device__ __forceinline__ uint32_t endless(const Pack<T, 8> &v) {
    constexpr int kWords = 8 * sizeof(T) / 4;
    constexpr uint32_t kOnes = std::is_same_v<T, float> ? 0x7f800000u : std::is_same_v<T, bf16> ? 0x7f807f80u : 0x7c007c00u;
    constexpr uint32_t kOne = std::is_same_v<T, float> ? 0x00800000u : std::is_same_v<T, bf16> ? 0x00800080u : 0x04000400u;
    uint32_t w[kWords], found = 0;
    __builtin_memcpy(w, &v, sizeof(w));
#pragma unroll
    for (int i = 0; i < kWords; i++) found |= (w[i] & kOnes) + kOne;
    return found & (sizeof(T) == 4 ? 0x80000000u : 0x80008000u);
}

// Rows of a chunk on their way from memory to a tile: the thread's vectors of 8 places
template <typename T, int W, int R, int THREADS>
struct Rows {
    static constexpr int kPer = W / 8, kLoads = (R * kPer + THREADS - 1) / THREADS, kApart = THREADS / kPer;      // rows from vector to vector
    static_assert(THREADS % kPer == 0 && (R * kPer % THREADS == 0 || kLoads == 1));
    static constexpr bool kAll = R * kPer % THREADS == 0;      // whether all threads have a vector
    Pack<T, 8> v[kLoads];

    // true where a value is an infinity or a NaN
    template <typename E, int P, bool ORDERED>
    __device__ __forceinline__ bool store(Tile<E, P, W, R, ORDERED> &tile) const {
        uint32_t odd = 0;
        const int r0 = (int)threadIdx.x / kPer, c = (int)threadIdx.x % kPer * 8;
#pragma unroll
        for (int k = 0; k < kLoads; k++) {
            const int r = r0 + k * kApart;
            if (!kAll && r >= R) break;
            const Pack<T, 8> &u = v[k];
            odd |= endless<T>(u);
            if constexpr (std::is_same_v<T, E>) tile.put(0, r, c, u);
            else {
                Pack<E, 8> hi, lo;
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    hi.v[e] = (E)(float)u.v[e];
                    lo.v[e] = (E)((float)u.v[e] - (float)hi.v[e]);
                }
                tile.put(0, r, c, hi);
                tile.put(1, r, c, lo);
            }
        }
        return odd != 0;
    }
};

// Where a thread finds them: places c0 .. c0 + W - 1 of `width`; zeros where there are none.  EVEN: the width is a multiple of 8, so that
// all vectors of 8 lie inside rows or behind them.
template <typename T, int W, int R, int THREADS, bool EVEN>
struct RowsOf {
    using To = Rows<T, W, R, THREADS>;
    const T *mine;                       // the thread's first element, were the chunk's first row the operand's
    int64_t step;
    int left;                            // places from the thread's first on
    bool full;                           // whether all threads have some, the whole of 8

    __device__ __forceinline__ RowsOf(const Operand &m, int32_t head, bool down, int c0, int width) {
        const int r = (int)threadIdx.x / To::kPer, c = c0 + (int)threadIdx.x % To::kPer * 8;
        step = down ? -m.ld : m.ld;
        mine = (const T *)m.at + (head / m.group) * m.hd + r * step + c;
        left = width - c;
        full = EVEN && To::kAll && width - c0 >= W;
    }
    // `count` rows from `row` on, upwards or downwards
    __device__ __forceinline__ void load(To &to, const Operand &m, int64_t row, int count) const {
        const T *from = mine + row * m.ld;
        const int r = (int)threadIdx.x / To::kPer;
        if (count == R && full) {
#pragma unroll
            for (int k = 0; k < To::kLoads; k++) to.v[k] = load_pack<T, 8>(from + k * To::kApart * step);
            return;
        }
#pragma unroll
        for (int k = 0; k < To::kLoads; k++) {
            to.v[k] = Pack<T, 8>{};
            const bool here = r + k * To::kApart < count;
            if constexpr (EVEN) {
                if (here && left > 0) to.v[k] = load_pack<T, 8>(from + k * To::kApart * step);
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (here && e < left) to.v[k].v[e] = from[k * To::kApart * step + e];
            }
        }
    }
};

}  // namespace attention
}  // namespace cpeval
