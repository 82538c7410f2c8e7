// Linear attention with a decay for each head: a recurrence whose state is a matrix,
//
//   S_t = gamma S_{t-1} + k_t^T v_t,   o_t = scale q_t S_t,   gamma = exp(log_decay) of the head
//
// in chunks of 32 or 64 rows, which makes it matrix products: with S the state that enters a chunk and i, j its rows,
//
//   o_i = scale (gamma^(i+1) q_i S + sum_{j <= i} gamma^(i-j) (q_i . k_j) v_j)
//   S'  = gamma^n S + sum_j gamma^(n-1-j) k_j^T v_j
//
// A wavefront owns 16 or 32 columns of S, in registers, and walks along the rows; q, k and v of a chunk lie in LDS.  The scores, of which only
// the tiles on and below the diagonal are computed, are shared out among the wavefronts.
//
// What bounds a pass of bf16 heads of 128: 65,536 rows of 16 heads in 377 to 426 us, 1.07 GB at 2.5 to 2.8 TB/s.  With two wavefronts a SIMD, which is
// what registers leave room for, loads, LDS and products of one hide too little of the other's: the matrix units are busy for 30% of the
// time, and wavefronts wait for their turn to issue for 29% of theirs.
//
// The gradient is three such passes.  With D_t = gamma D_{t+1} + scale q_t^T do_t the gradient of S_t,
//   dq_t = scale do_t S_t^T (the pass with do, v, k in the places of q, k, v),   dv_t = k_t D_t and dk_t = v_t D_t^T (from the last
//   row on, with k, q, do and v, do, q),   dlog_decay = sum_t <D_t, gamma S_{t-1}>, which the last two add up.
//
// Where sequences and heads do not fill the chip, the rows are cut into segments: each segment's effect on the state first, then the
// states that enter them, segment by segment, then the outputs.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "linear_attention.hpp"

namespace cpeval {
namespace attention {

namespace {

// up to 4 neighbouring results, rounded once
template <typename T>
__device__ __forceinline__ void put(T *to, f32x4 o, float scale, int count) {
    Pack<T, 4> v;
#pragma unroll
    for (int e = 0; e < 4; e++) v.v[e] = (T)(o[e] * scale);
    if (count >= 4) store_pack<T, 4>(to, v);
    else {
#pragma unroll
        for (int e = 0; e < 3; e++)
            if (e < count) to[e] = v.v[e];
    }
}

// ---- the pass ----------------------------------------------------------------------------------------

// kOut: outputs; kEffect: a segment's effect on the state alone.  The other two add to outputs their part of the decays' gradient.  That is, for
// every chunk with S the state that enters it, X the gradient of the state behind it and P the scores,
//   sum_i (i + 1) q_i . dq_i by S + sum_ij (i - j) P_ij (q_i . k_j) + sum_j (n - 1 - j) k_j . dk_j by X + n gamma^n <S, X>
// kGrad: the first two in the pass for dq, and the last by carrying R' = gamma^n (R + n S) along, as sum_i q_i . dq_i by R and what R
// ends in times its gradient.  kLeave: the third in the pass for dk.
enum Kind { kOut, kEffect, kGrad, kLeave };

// NT times 16 columns of a state, all of its rows, in a wavefront's registers: lane l has column l % 16, rows 16 k + 4 (l / 16) + 0..3
template <int KB, int NT>
struct State {
    f32x4 at[NT][2 * KB];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int t = 0; t < NT; t++)
#pragma unroll
            for (int k = 0; k < 2 * KB; k++) at[t][k] = f32x4{0, 0, 0, 0};
    }
    // (where the lane's first element lies is hidden from the compiler, which else keeps the addresses of all of them, and whether they
    // are there, in registers throughout the pass)
    template <typename F>
    __device__ __forceinline__ void each(const Pass &p, int64_t index, int32_t head, int col, int g, F f) {
        int row0 = 4 * g;
        asm volatile("" : "+v"(row0));
        const int64_t base = (index * p.heads + head) * ((int64_t)p.wa * p.wb);
        const int across = p.transposed ? p.wa : 1, down = p.transposed ? 1 : p.wb;
#pragma unroll
        for (int t = 0; t < NT; t++)
#pragma unroll
            for (int k = 0; k < 2 * KB; k++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int row = row0 + 16 * k + e, c = col + 16 * t;
                    if (row < p.wa && c < p.wb) at[t][k][e] = f(at[t][k][e], base + (c * across + row * down));
                }
    }
    __device__ __forceinline__ void load(const Pass &p, const float *from, int64_t index, int32_t head, int col, int g) {
        zero();
        each(p, index, head, col, g, [&](float, int64_t i) { return from[i]; });
    }
    __device__ __forceinline__ void store(const Pass &p, float *to, int64_t index, int32_t head, int col, int g) {
        each(p, index, head, col, g, [&](float v, int64_t i) { return to[i] = v; });
    }
    __device__ __forceinline__ double dot(const Pass &p, const float *with, int64_t index, int32_t head, int col, int g) {
        double sum = 0;
        each(p, index, head, col, g, [&](float v, int64_t i) { return sum += (double)(v * with[i]), v; });
        return sum;
    }
    __device__ __forceinline__ void decay(const Fade &fade) {
#pragma unroll
        for (int t = 0; t < NT; t++)
#pragma unroll
            for (int k = 0; k < 2 * KB; k++)
#pragma unroll
                for (int e = 0; e < 4; e++) at[t][k][e] = faded(at[t][k][e], fade);
    }
    __device__ __forceinline__ void add(const State &s, float by) {
#pragma unroll
        for (int t = 0; t < NT; t++)
#pragma unroll
            for (int k = 0; k < 2 * KB; k++)
#pragma unroll
                for (int e = 0; e < 4; e++) at[t][k][e] = fmaf(s.at[t][k][e], by, at[t][k][e]);
    }
};

// KB: blocks of 32 that the state's rows fill; NT: of 16 columns that a wavefront has; WAVES: of a workgroup; R: rows of a chunk;
// EVEN: widths are multiples of 8
template <typename T, int KB, int NT, int WAVES, int R, Kind kind, bool EVEN>
__global__ __launch_bounds__(WAVES * kWave, R == 32 && KB == 2 && kind != kGrad ? 4 : 2) void pass_kernel(Pass p, float *effect, Gain *gain) {
    using F = Form<T>;
    using E = typename F::E;
    constexpr int P = F::kPlanes, PS = F::kSplit;
    constexpr bool kAhead = kind == kEffect || (kind == kGrad ? KB == 2 && sizeof(T) == 2 : KB * NT != 8 || KB == 8);
    constexpr int kThreadsHere = WAVES * kWave, kWide = 16 * NT * WAVES, IT = R / 16, JB = R / 32;
    __shared__ Tile<E, P, 32 * KB, R, false> b_tile;
    __shared__ Tile<E, P, kWide, R, false> x_tile;
    // Scores [row][place] take the place of a's rows (and d's) when these have been read: three parts and the rows together would leave
    // room for one workgroup of bf16 heads of 128 a compute unit.
    using Scores = Tile<E, PS, kind == kEffect ? 8 : R, kind == kEffect ? 1 : R, true>;
    using First = Tile<E, P, kind == kEffect ? 8 : 32 * KB, kind == kEffect ? 1 : R, true>;
    using Third = Tile<E, P, kind == kGrad ? kWide : 8, kind == kGrad ? R : 1, true>;
    constexpr size_t kFirst = sizeof(First) + (kind == kGrad ? sizeof(Third) : 0);
    __shared__ __attribute__((aligned(16))) char shared_[kFirst > sizeof(Scores) ? kFirst : sizeof(Scores)];
    First &a_tile = *(First *)shared_;
    Third &d_tile = *(Third *)(shared_ + (kind == kGrad ? sizeof(First) : 0));
    Scores &s_tile = *(Scores *)shared_;
    __shared__ int odd[2];

    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), l = lane % 16, g = lane / 16;
    const uint32_t group = group_number();
    const int32_t slice = group % p.slices, head = group / p.slices % p.heads, seg = group / p.slices / p.heads;
    if (seg >= p.segments) return;                     // (the whole workgroup)
    const int c0 = slice * kWide, mine = 16 * NT * wave, col = c0 + mine + l;
    const Decay lg = decay_of(p.log_decay ? p.log_decay[head] : 0.0f);

    int64_t lo, hi;
    segment_of(p, seg, lo, hi);
    if (threadIdx.x == 0) odd[0] = odd[1] = 0;
    __syncthreads();                                   // (before another wavefront finds an infinity in its first rows)
    double decay_sum = 0;
    int turn = 0;
    State<KB, NT> s, r;
    if constexpr (kind == kEffect) {
        // only the sequence that goes on behind the segment: the last piece in the order of the pass, which is the first one seen from there
        s.zero();
        bool ends = true, whole = false;
        if (lo < hi) {
            Pass turned = p;
            turned.back = !p.back;
            const Piece last = piece_at(turned, lo, hi);
            ends = last.starts, whole = !last.ends;    // (its end and its start, seen from there)
            lo = last.lo, hi = last.hi;
        }
        if (threadIdx.x == 0 && slice == 0) gain[(int64_t)seg * p.heads + head] = {fade_of(lg, (int)(hi - lo)), !whole || ends};
        if (ends) lo = hi;
    }
    // What does not change from chunk to chunk: the decays between a score's rows, of this wavefront's tiles, into rows from before
    // the chunk, and from rows to its end
    constexpr int kTiles = IT * (IT + 1) / 2, kMine = (kTiles + WAVES - 1) / WAVES;
    float apart_[kMine][4], in_[IT], out_[JB][8];
    const auto tile_of = [&](int k, int &it, int &jt) {
        const int tile = wave + k * WAVES;
        it = 0;
#pragma unroll
        for (int n = 1; n < IT; n++) it += tile >= n * (n + 1) / 2;
        jt = tile - it * (it + 1) / 2;
        return tile < kTiles;
    };
    if constexpr (kind != kEffect) {
#pragma unroll
        for (int k = 0; k < kMine; k++) {
            int it, jt;
            if (!tile_of(k, it, jt)) continue;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int apart = 16 * (it - jt) + l - 4 * g - e;
                apart_[k][e] = apart < 0 ? 0.0f : power(lg, apart) * p.s_in;
            }
        }
#pragma unroll
        for (int it = 0; it < IT; it++) in_[it] = power(lg, 16 * it + l + 1 - p.shift);
    }
    const auto behind = [&](int jb, int e, int count) { return max(count - 1 - (32 * jb + 16 * (e / 4) + 4 * g + e % 4), 0); };
#pragma unroll
    for (int jb = 0; jb < JB; jb++)
#pragma unroll
        for (int e = 0; e < 8; e++) out_[jb][e] = power(lg, behind(jb, e, R) + p.shift) * p.s_in;
    const Fade wane_ = fade_of(lg, R);

    const RowsOf<T, 32 * KB, R, kThreadsHere, EVEN> a_rows(p.a, head, p.back, 0, p.wa), b_rows(p.b, head, p.back, 0, p.wa);
    const RowsOf<T, kWide, R, kThreadsHere, EVEN> x_rows(p.x, head, p.back, c0, p.wb), d_rows(p.d, head, p.back, c0, p.wb);
    while (lo < hi) {
        const Piece piece = piece_at(p, lo, hi);
        int64_t left = piece.hi - piece.lo, row = p.back ? piece.hi - 1 : piece.lo;
        if (piece.starts && p.init) s.load(p, p.init, piece.seq, head, col, g);
        else if (kind != kEffect && !piece.starts && p.enter) s.load(p, p.enter, seg, head, col, g);
        else s.zero();
        if constexpr (kind == kGrad) r.zero();
        // (from the last row on, the first chunk is the shorter one, so that all passes have the same)
        int next = kind != kEffect && p.last_first ? (int)((left - 1) % R) + 1 : (int)min((int64_t)R, left);
        Rows<T, 32 * KB, R, kThreadsHere> a_now, b_now;
        Rows<T, kWide, R, kThreadsHere> x_now, d_now;
        const auto fetch = [&] {
            x_rows.load(x_now, p.x, row, next);
            b_rows.load(b_now, p.b, row, next);
            if constexpr (kind != kEffect) a_rows.load(a_now, p.a, row, next);
            if constexpr (kind == kGrad) d_rows.load(d_now, p.d, row, next);
        };
        if (kAhead) fetch();
        int single = 0;                                // rows of a chunk that go one by one, their part of the decays' gradient being done
        while (left > 0) {
            if (!kAhead) fetch();
            const bool found = x_now.store(x_tile);
            b_now.store(b_tile);
            if constexpr (kind != kEffect) {
                a_now.store(a_tile);
                if (found) odd[turn] = 1;
            }
            if constexpr (kind == kGrad) d_now.store(d_tile);
            __syncthreads();
            bool sums = true, rest = true;             // what is done: the decays' gradient; all else
            if constexpr (kind != kEffect) {
                // An infinity or a NaN in x would pass, times a score of 0, to the rows before its own: such chunks go row by row.  (kGrad: behind the sums
                // of the chunk as a whole, which kLeave's are cut like.)
                const bool bad = __builtin_amdgcn_readfirstlane(odd[turn]);
                turn ^= 1;
                if (threadIdx.x == 0) odd[turn] = 0;
                if constexpr (kind == kGrad) {
                    sums = single == 0, rest = !(bad && next > 1);
                } else if (bad && next > 1) {
                    next = 1;
                    __syncthreads();
                    if (kAhead) fetch();
                    continue;
                }
            }
            const int count = next;
            const int64_t here = row;
            if (rest) {
                left -= count;
                row += p.back ? -count : count;
                if (single > 0) single--;
            } else single = count;
            next = single > 0 ? 1 : (int)min((int64_t)R, left);
            if constexpr (kind == kEffect) {
                if (left > 0) fetch();
            }

            f32x4 o[NT][IT];
            if constexpr (kind != kEffect) {
                // scores of rows i (lanes) and j (places): the tiles on and below the diagonal, shared out, in registers until a's rows have been read
                f32x4 score[kMine];
#pragma unroll
                for (int m = 0; m < kMine; m++) {
                    int it, jt;
                    if (!tile_of(m, it, jt)) continue;
                    f32x4 c = {0, 0, 0, 0};
#pragma unroll
                    for (int k0 = 0; k0 < KB; k0 += 4) {
                        Frag<E, P> bf[4], af[4];
#pragma unroll
                        for (int k = 0; k < 4; k++)
                            if (k0 + k < KB) bf[k] = b_tile.along(16 * jt, k0 + k, lane), af[k] = a_tile.along(16 * it, k0 + k, lane);
                        asked();
#pragma unroll
                        for (int k = 0; k < 4; k++)
                            if (k0 + k < KB) c = product<true>(bf[k], af[k], c);
                    }
#pragma unroll
                    for (int e = 0; e < 4; e++) c[e] = it == jt && 4 * g + e > l ? 0.0f : c[e] * apart_[m][e];     // (what lies above the diagonal is not looked at)
                    if constexpr (kind == kGrad) {
                        f32x4 other = {0, 0, 0, 0};
#pragma unroll
                        for (int k0 = 0; k0 < kWide / 32; k0 += 2) {
                            Frag<E, P> xs[2], ds[2];
#pragma unroll
                            for (int k = 0; k < 2; k++) xs[k] = x_tile.along(16 * jt, k0 + k, lane), ds[k] = d_tile.along(16 * it, k0 + k, lane);
                            asked();
#pragma unroll
                            for (int k = 0; k < 2; k++) other = product<true>(xs[k], ds[k], other);
                        }
                        float sum = 0;
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            const int apart = 16 * (it - jt) + l - 4 * g - e;
                            if (apart > 0 && 16 * it + l < count) sum += (float)apart * c[e] * other[e];      // (0 of no row times a NaN is one)
                        }
                        if (sums) decay_sum += (double)(sum * p.s_out);
                    }
                    score[m] = c;
                }
                // what the state that enters gives, 32 of its rows at a time
                f32x4 more[NT][kind == kGrad ? IT : 1];
#pragma unroll
                for (int t = 0; t < NT; t++)
#pragma unroll
                    for (int it = 0; it < IT; it++) {
                        o[t][it] = f32x4{0, 0, 0, 0};
                        if constexpr (kind == kGrad) more[t][it] = f32x4{0, 0, 0, 0};
                    }
                Frag<E, P> af[2][IT];
                const auto ask = [&](int k) {
#pragma unroll
                    for (int it = 0; it < IT; it++) af[k % 2][it] = a_tile.along(16 * it, k, lane);
                };
                ask(0);
#pragma unroll
                for (int k = 0; k < KB; k++) {
                    if (k + 1 < KB) ask(k + 1);
                    asked();
#pragma unroll
                    for (int t = 0; t < NT; t++) {
                        Frag<E, PS> sf;
                        split(s.at[t][2 * k], s.at[t][2 * k + 1], sf);
                        products<true>(af[k % 2], sf, o[t]);
                        if constexpr (kind == kGrad) {
                            split(r.at[t][2 * k], r.at[t][2 * k + 1], sf);
                            products<true>(af[k % 2], sf, more[t]);
                        }
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; t++) {
                    const int c = c0 + mine + 16 * t + 4 * g;
#pragma unroll
                    for (int it = 0; it < IT; it++) {
#pragma unroll
                        for (int e = 0; e < 4; e++) o[t][it][e] *= in_[it];
                        if constexpr (kind == kGrad || kind == kLeave) {
                            const int i = 16 * it + l;
                            // (a sequence's last row, whose state no decay follows, has no part even if it holds a NaN)
                            if (i >= count || c >= p.wb || !sums || (kind == kLeave && i == 0)) continue;
                            const T *from = (const T *)p.d.at + (here + (p.back ? -i : i)) * p.d.ld + (head / p.d.group) * p.d.hd + c;
                            float sum = 0;
                            Pack<T, 4> with{};
                            if constexpr (EVEN) with = load_pack<T, 4>(from);
                            else {
#pragma unroll
                                for (int e = 0; e < 4; e++)
                                    if (c + e < p.wb) with.v[e] = from[e];
                            }
#pragma unroll
                            for (int e = 0; e < 4; e++) {
                                const float one = kind == kGrad ? fmaf(more[t][kind == kGrad ? it : 0][e], in_[it], (float)(i + 1) * o[t][it][e]) : (float)i * o[t][it][e];
                                sum = fmaf((float)with.v[e], one, sum);
                            }
                            decay_sum += (double)(sum * p.s_out);
                        }
                    }
                }
                __syncthreads();
#pragma unroll
                for (int m = 0; m < kMine; m++) {
                    int it, jt;
                    if (!tile_of(m, it, jt)) continue;
                    s_tile.keep(16 * it + l, 16 * jt + 4 * g, score[m]);
                    // (right of a diagonal's tile, in its block of 32)
                    if (it == jt && it % 2 == 0) s_tile.keep(16 * it + l, 16 * jt + 16 + 4 * g, f32x4{0, 0, 0, 0});
                }
                __syncthreads();
            }
            Frag<E, P> xf[NT][JB];
#pragma unroll
            for (int t = 0; t < NT; t++)
#pragma unroll
                for (int jb = 0; jb < JB; jb++) xf[t][jb] = x_tile.across(mine + 16 * t, jb, lane);
            if constexpr (kind != kEffect) {
                // and what its own rows give
#pragma unroll
                for (int jb = 0; jb < JB; jb++)
#pragma unroll
                    for (int i0 = 2 * jb; i0 < IT; i0 += 2) {
                        Frag<E, PS> sc[2];
#pragma unroll
                        for (int k = 0; k < 2; k++) sc[k] = s_tile.along(16 * (i0 + k), jb, lane);
                        asked();
#pragma unroll
                        for (int t = 0; t < NT; t++)
#pragma unroll
                            for (int k = 0; k < 2; k++) o[t][i0 + k] = product(xf[t][jb], sc[k], o[t][i0 + k]);
                    }
#pragma unroll
                for (int t = 0; t < NT; t++) {
                    const int c = c0 + mine + 16 * t + 4 * g;
                    const int64_t to = (here + (p.back ? -l : l)) * p.ldo + head * p.hdo + c, step = (p.back ? -16 : 16) * p.ldo;
                    const int places = EVEN ? 4 : p.wb - c;
                    if (c < p.wb && rest) {
#pragma unroll
                        for (int it = 0; it < IT; it++) {
                            if (16 * it + l >= count) continue;
                            if (p.wide) put((float *)p.o + to + it * step, o[t][it], p.s_out, places);
                            else put((T *)p.o + to + it * step, o[t][it], p.s_out, places);
                        }
                    }
                }
            }

            // The next chunk is on its way while the state is computed, where there are registers for it.  (Where some go to scratch memory, whose
            // loads wait for all others before them, it costs more than it gives: 8 sequences of 4,096 rows of 16 heads of 128 in bf16 1,242 us for 1,105,
            // forward and backward; where there are, 52,710 rows of 6 heads of 48 keys and 80 values in fp16 773 for 802.  1,000,000 rows of 4 heads of 64
            // in bf16 3.00 ms either way.)
            if constexpr (kAhead && kind != kEffect) {
                if (left > 0) fetch();
                asked();
            }

            // the state behind the chunk
            Fade wane = wane_;
            if (count != R) wane = fade_of(lg, count);
            if constexpr (kind == kGrad) {
                if (sums) {
                    r.add(s, (float)count);
                    r.decay(wane);
                }
                if (!rest) {
                    __syncthreads();
                    continue;
                }
            }
            s.decay(wane);
#pragma unroll
            for (int jb = 0; jb < JB; jb++) {
                float by[8];
#pragma unroll
                for (int e = 0; e < 8; e++) by[e] = out_[jb][e];
                if (count != R) {
#pragma unroll
                    for (int e = 0; e < 8; e++) by[e] = power(lg, behind(jb, e, count) + p.shift) * p.s_in;      // (rows behind the chunk's are zeros)
                }
                Frag<E, PS> vf[NT];
#pragma unroll
                for (int t = 0; t < NT; t++) {
                    float v[8];
                    values(xf[t][jb], v);
#pragma unroll
                    for (int e = 0; e < 8; e++) v[e] *= by[e];
                    split(v, vf[t]);
                }
                constexpr int kGroup = 4;
#pragma unroll
                for (int k0 = 0; k0 < 2 * KB; k0 += kGroup) {
                    Frag<E, P> bf[kGroup];
#pragma unroll
                    for (int k = 0; k < kGroup; k++) bf[k] = b_tile.across(16 * (k0 + k), jb, lane);
                    asked();
#pragma unroll
                    for (int t = 0; t < NT; t++) products(bf, vf[t], &s.at[t][k0]);
                }
            }
            __syncthreads();
        }
        if constexpr (kind == kOut) {
            if (piece.ends && p.last) s.store(p, p.last, piece.seq, head, col, g);
        }
        if constexpr (kind == kGrad) {
            if (piece.ends) {
                if (p.dlast) decay_sum += r.dot(p, p.dlast, piece.seq, head, col, g);
            } else if (p.denter) decay_sum += r.dot(p, p.denter, seg, head, col, g);
        }
        if (p.back) hi = piece.lo;
        else lo = piece.hi;
    }
    if constexpr (kind == kEffect) s.store(p, effect, seg, head, col, g);
    if constexpr (kind == kGrad || kind == kLeave) {
        __shared__ double sums[WAVES];
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) decay_sum += __shfl_xor(decay_sum, off);
        if (lane == 0) sums[wave] = decay_sum;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < WAVES; w++) decay_sum += sums[w];
            p.part[head * p.part_step + (int64_t)seg * p.slices + slice] = decay_sum;
        }
    }
}

// States that enter the segments, from their effects, in place and in the order of the pass: E' = gamma^n E + U.  Where a sequence began, the
// state before it is dropped, whatever it holds; a gamma^n of 0 does not do that, as 0 times a NaN is one.  (gamma^n in 32 bits is off by
// the same in every segment: by up to 2e-5 of a state after 1,024.)  Sixteen segments' loads are under way at once: 256 segments of 4
// heads of 64 x 64 in 43 us, 88 with one segment's alone.
template <int V>
__global__ __launch_bounds__(kThreads) void enter_kernel(float *at, const Gain *gain, int32_t segments, int32_t heads, int32_t size, bool back) {
    const int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * V;
    if (i >= size) return;
    const int32_t head = blockIdx.y;
    Pack<float, V> e;
#pragma unroll
    for (int k = 0; k < V; k++) e.v[k] = 0.0f;
    constexpr int kAhead = 16;                         // segments whose effects are under way at once
    const auto segment = [&](int32_t n) { return (int64_t)(back ? segments - 1 - n : n) * heads + head; };
    for (int32_t n0 = 0; n0 < segments; n0 += kAhead) {
        Pack<float, V> u[kAhead];
        Gain by[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; a++) {
            const int32_t n = min(n0 + a, segments - 1);
            u[a] = load_pack<float, V>(at + segment(n) * size + i);
            by[a] = gain[segment(n)];
        }
#pragma unroll
        for (int a = 0; a < kAhead; a++) {
            if (n0 + a >= segments) break;
            store_pack<float, V>(at + segment(n0 + a) * size + i, e);
#pragma unroll
            for (int k = 0; k < V; k++) e.v[k] = by[a].drops ? u[a].v[k] : faded(e.v[k], by[a].fade) + u[a].v[k];
        }
    }
}

// Pointers that do not rise from 0, or beyond the rows
__global__ __launch_bounds__(kThreads) void check_kernel(const int32_t *ptr, int32_t num_seq, int64_t rows, int32_t *status) {
    __shared__ int bad;
    if (threadIdx.x == 0) bad = ptr[0] != 0 || ptr[num_seq] > rows;
    __syncthreads();
    bool mine = false;
    for (int64_t s = threadIdx.x; s < num_seq; s += kThreads) mine |= ptr[s + 1] < ptr[s];
    if (mine) bad = 1;
    __syncthreads();
    if (threadIdx.x == 0) *status = bad ? CP_STATUS_BAD_SEQUENCE : CP_STATUS_OK;
}

// A sequence without rows ends in the state that it begins with
__global__ __launch_bounds__(kThreads) void empty_kernel(const int32_t *ptr, int64_t len, int32_t num_seq, int64_t state, const float *from, float *to) {
    for (int64_t s = blockIdx.x; s < num_seq; s += gridDim.x) {
        if (ptr ? ptr[s + 1] > ptr[s] : len > 0) continue;
        for (int64_t i = (int64_t)blockIdx.y * kThreads + threadIdx.x; i < state; i += (int64_t)gridDim.y * kThreads)
            to[s * state + i] = from ? from[s * state + i] : 0.0f;
    }
}

// Gradients of a head's keys or values from those of the heads that share it, in their order; a wavefront a row, V neighbouring values a lane
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void share_kernel(const float *part, const int32_t *ptr, int32_t num_seq, int64_t rows, int32_t heads, int32_t group,
                                                         int32_t width, T *to, int64_t ld, int64_t hd) {
    const int64_t total = ptr ? min((int64_t)max(ptr[num_seq], 0), rows) : rows;
    const int32_t line = heads / group * width / V;
    for (int64_t row = (int64_t)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave; row < total; row += (int64_t)gridDim.x * (kThreads / kWave))
        for (int32_t i = threadIdx.x % kWave; i < line; i += kWave) {
            const int32_t h = i * V / width, c = i * V % width;
            const float *from = part + (row * heads + (int64_t)h * group) * width + c;
            Pack<float, V> sum = load_pack<float, V>(from);
            for (int32_t k = 1; k < group; k++) {
                const Pack<float, V> one = load_pack<float, V>(from + (int64_t)k * width);
#pragma unroll
                for (int e = 0; e < V; e++) sum.v[e] += one.v[e];
            }
            Pack<T, V> put;
#pragma unroll
            for (int e = 0; e < V; e++) put.v[e] = (T)sum.v[e];
            store_pack<T, V>(to + row * ld + h * hd + c, put);
        }
}

__global__ __launch_bounds__(kThreads) void decay_kernel(const double *part, int64_t each, float *to) {
    __shared__ double sums[kThreads];
    double sum = 0;
    for (int64_t i = threadIdx.x; i < each; i += kThreads) sum += part[blockIdx.x * each + i];
    sums[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kThreads; i++) sum += sums[i];
        to[blockIdx.x] = (float)sum;
    }
}

// ---- one more row of every sequence --------------------------------------------------------------------

struct Step {
    int32_t count, heads, wk, wv, num_slots;
    Operand q, k, v;
    const float *log_decay;
    float scale;
    float *state;
    const int32_t *slots;
    void *o;
    int64_t ldo, hdo;
    int32_t *status;
};

// A workgroup has the state of one head of one sequence; a thread V neighbouring columns of every few rows.  It is read once and written
// once, which is all there is to it: 512 sequences of 16 heads of 128 x 128 in 217 us, 1.08 GB at 5.0 TB/s, the rate of a copy.
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void step_kernel(Step p) {
    __shared__ float sums[kThreads * V], kq[2][256];
    const int64_t unit = group_number();
    const int32_t head = (int32_t)(unit % p.heads);
    const int64_t seq = unit / p.heads;
    if (seq >= p.count) return;
    const int32_t slot = p.slots ? p.slots[seq] : (int32_t)seq;
    const bool bad = slot >= p.num_slots;
    if (bad && p.slots && threadIdx.x == 0 && head == 0) atomicOr(p.status, CP_STATUS_BAD_SLOT);
    T *o = (T *)p.o + seq * p.ldo + head * p.hdo;
    if (slot < 0 || bad) {
        for (int c = threadIdx.x; c < p.wv; c += kThreads) o[c] = (T)0.0f;
        return;
    }
    const T *q = (const T *)p.q.at + seq * p.q.ld + (head / p.q.group) * p.q.hd;
    const T *k = (const T *)p.k.at + seq * p.k.ld + (head / p.k.group) * p.k.hd;
    const T *v = (const T *)p.v.at + seq * p.v.ld + (head / p.v.group) * p.v.hd;
    for (int c = threadIdx.x; c < p.wk; c += kThreads) kq[0][c] = (float)k[c], kq[1][c] = (float)q[c];
    const Fade fade = fade_of(decay_of(p.log_decay ? p.log_decay[head] : 0.0f), 1);      // (4,000 steps of gamma in 32 bits: 1e-4 off)
    const int lanes = (p.wv + V - 1) / V, side = kThreads / lanes;      // (wv is a multiple of V; lanes <= 256)
    const int mine = threadIdx.x % lanes, first = threadIdx.x / lanes;
    float *state = p.state + ((int64_t)slot * p.heads + head) * ((int64_t)p.wk * p.wv) + mine * V;
    float value[V], sum[V];
#pragma unroll
    for (int e = 0; e < V; e++) value[e] = (float)v[mine * V + e], sum[e] = 0.0f;
    __syncthreads();
    if (first < side) {
#pragma unroll 8
        for (int row = first; row < p.wk; row += side) {
            Pack<float, V> s = load_pack<float, V>(state + (int64_t)row * p.wv);
#pragma unroll
            for (int e = 0; e < V; e++) {
                s.v[e] = fmaf(kq[0][row], value[e], faded(s.v[e], fade));
                sum[e] = fmaf(kq[1][row], s.v[e], sum[e]);
            }
            store_pack<float, V>(state + (int64_t)row * p.wv, s);
        }
    }
#pragma unroll
    for (int e = 0; e < V; e++) sums[threadIdx.x * V + e] = sum[e];
    __syncthreads();
    for (int c = threadIdx.x; c < p.wv; c += kThreads) {
        float all = 0.0f;
        for (int i = 0; i < side; i++) all += sums[i * lanes * V + c];
        o[c] = (T)(all * p.scale);
    }
}

__global__ void set_status_kernel(int32_t *status, int32_t value) { *status = value; }

// ---- host --------------------------------------------------------------------------------------------

constexpr int kMaxWidth = CP_ATTENTION_MAX_WIDTH, kMaxHeads = CP_ATTENTION_MAX_HEADS;

// Segments: workgroups enough to fill the chip once, two a compute unit, and twice as many for heads of up to 64, of which four fit; of 128 rows at
// least.  The same for all types and for both directions, since the backward pass reads the states that the forward call kept.  (Forward and
// backward in bf16: 1,000,000 rows of 4 heads of 64 3.00 ms, 3.30 with half as many, 3.12 with twice; 8 sequences of 4,096 rows of 16 heads of 128 1.10
// ms, 1.35 with half as many, 1.25 with twice, whose states cost more than the fuller chip gives.)
struct Cut {
    int64_t seg_rows;
    int32_t parts, segments;
    bool split;                          // whether a sequence may be cut
};
constexpr int64_t kLeast = 128;

Cut cut_of(int64_t rows, int32_t num_seq, bool packed, int32_t heads, int32_t wk, int32_t wv) {
    const int64_t kWanted = std::max(wk, wv) <= 64 ? 1024 : 512;
    const int64_t len = packed ? rows : rows / num_seq;
    const int64_t units = (int64_t)heads * (packed ? 1 : num_seq);
    int64_t parts = std::max<int64_t>(1, std::min(kWanted / units, len / kLeast));
    Cut c;
    c.seg_rows = std::max<int64_t>((len + parts - 1) / parts, 1);
    c.seg_rows = (c.seg_rows + 63) / 64 * 64;
    parts = std::max<int64_t>(1, (len + c.seg_rows - 1) / c.seg_rows);
    c.parts = (int32_t)parts;
    c.segments = (int32_t)(packed ? parts : parts * num_seq);
    c.split = parts > 1;
    return c;
}

// Columns that a workgroup takes: 64 where there are no more, else 128
int32_t columns_of(int32_t wa, int32_t wb) { return wb > 64 || wa > 128 ? 128 : 64; }
int32_t slices_of(int32_t wa, int32_t wb) { return (wb + columns_of(wa, wb) - 1) / columns_of(wa, wb); }

template <typename T, int KB, int COLUMNS, bool EVEN>
int run_sized(Kind kind, const Pass &p, float *effect, Gain *gain, hipStream_t st) {
    // Columns a wavefront: 32 of bf16 heads of up to 128, whose operands then serve two products (65,536 rows of 16 heads of 128 forward 532 us, 581 with 16;
    // 8 x 4,096 rows forward and backward 1.10 ms, 1.22).  The other types' operands, of two or three parts or in 32 bits, leave no registers for it.
    // Rows of a chunk: 64, so that a state is read and split once for as many, but for three.  bf16 heads of up to 64: of 32 rows four workgroups fit a
    // compute unit (1,000,000 rows of 4 heads of 64 3.00 ms, 3.24 with 64).  fp16 and float heads whose states have 65 to 128 rows and up to 64 columns:
    // tiles of 64 rows leave LDS for one workgroup (heads of 48 keys and 80 values, 52,710 rows of 6, 773 us, 943 with 64).  And those of more than
    // 128 rows, whose tiles of 64 do not fit at all.
    constexpr bool kHalf = std::is_same_v<T, bf16>;
    constexpr int R = (kHalf && KB == 2 && COLUMNS == 64) || (!kHalf && (KB == 8 || (KB == 4 && COLUMNS == 64))) ? 32 : 64;
    constexpr int NT = COLUMNS == 128 && kHalf && KB < 8 ? 2 : 1, WAVES = COLUMNS / 16 / NT;
    if (kind == kGrad) {       // (two states: 16 columns a wavefront)
        hipLaunchKernelGGL((pass_kernel<T, KB, 1, COLUMNS / 16, R, kGrad, EVEN>), grid_of((int64_t)p.segments * p.heads * p.slices), dim3(COLUMNS * 4), 0, st, p,
                           effect, gain);
        return launched();
    }
    auto *kernel = kind == kOut      ? pass_kernel<T, KB, NT, WAVES, R, kOut, EVEN>
                   : kind == kEffect ? pass_kernel<T, KB, NT, WAVES, R, kEffect, EVEN>
                                     : pass_kernel<T, KB, NT, WAVES, R, kLeave, EVEN>;
    hipLaunchKernelGGL(kernel, grid_of((int64_t)p.segments * p.heads * p.slices), dim3(WAVES * kWave), 0, st, p, effect, gain);
    return launched();
}

int run(Kind kind, int type, Pass p, float *effect, Gain *gain, hipStream_t st) {
    const bool even = p.wa % 8 == 0 && p.wb % 8 == 0, wide = columns_of(p.wa, p.wb) == 128;
    p.slices = slices_of(p.wa, p.wb);
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        if (p.wa > 128) return even ? run_sized<T, 8, 128, true>(kind, p, effect, gain, st) : run_sized<T, 8, 128, false>(kind, p, effect, gain, st);
        if (wide && p.wa > 64) return even ? run_sized<T, 4, 128, true>(kind, p, effect, gain, st) : run_sized<T, 4, 128, false>(kind, p, effect, gain, st);
        if (wide) return even ? run_sized<T, 2, 128, true>(kind, p, effect, gain, st) : run_sized<T, 2, 128, false>(kind, p, effect, gain, st);
        if (p.wa > 64) return even ? run_sized<T, 4, 64, true>(kind, p, effect, gain, st) : run_sized<T, 4, 64, false>(kind, p, effect, gain, st);
        return even ? run_sized<T, 2, 64, true>(kind, p, effect, gain, st) : run_sized<T, 2, 64, false>(kind, p, effect, gain, st);
    });
}

// the states that enter the pass's segments, into `at`
int run_enter(int type, const Pass &p, float *at, Gain *gain, hipStream_t st) {
    const int rc = run(kEffect, type, p, at, gain, st);
    if (rc) return rc;
    const int32_t size = p.wa * p.wb;
    const int per = size % 4 == 0 ? 4 : 1;
    const dim3 grid((unsigned)((size + kThreads * per - 1) / (kThreads * per)), (unsigned)p.heads);
    hipLaunchKernelGGL(per == 4 ? enter_kernel<4> : enter_kernel<1>, grid, dim3(kThreads), 0, st, at, gain, p.segments, p.heads, size, p.back);
    return launched();
}

struct Shape {
    int64_t rows;
    int32_t num_seq;
    const int32_t *ptr;
    int32_t heads, kv_heads, wk, wv;
    int type;
};

int check(const Shape &s, int reverse) {
    if (!known_type(s.type) || (reverse != 0 && reverse != 1)) return CP_ERR_ARG;
    if (s.rows < 0 || s.rows > INT32_MAX || s.num_seq < 1 || s.heads < 1 || s.heads > kMaxHeads || s.kv_heads < 1 || s.heads % s.kv_heads != 0 ||
        s.wk < 1 || s.wk > kMaxWidth || s.wv < 1 || s.wv > kMaxWidth)
        return CP_ERR_SIZE;
    // (workgroups are counted in 32 bits)
    if (s.ptr ? s.num_seq == INT32_MAX : s.rows % s.num_seq != 0 || (int64_t)s.num_seq * s.heads > INT32_MAX / 8) return CP_ERR_SIZE;
    return CP_OK;
}

size_t state_floats(const Shape &s) { return (size_t)s.heads * s.wk * s.wv; }
// of the states that enter segments, and of their gains
size_t enter_bytes(const Shape &s, const Cut &c) { return c.split ? align_up(c.segments * state_floats(s) * sizeof(float)) : 0; }
size_t gain_bytes(const Shape &s, const Cut &c) { return c.split ? align_up((size_t)c.segments * s.heads * sizeof(Gain)) : 0; }
// (of the passes for dq and dk, both of width_k columns)
int64_t part_count(const Shape &s, const Cut &c) { return 2 * (int64_t)c.segments * slices_of(s.wv, s.wk); }
size_t part_bytes(const Shape &s, const Cut &c) { return align_up((size_t)s.heads * part_count(s, c) * sizeof(double)); }
size_t share_bytes(const Shape &s) { return s.heads == s.kv_heads ? 0 : align_up((size_t)s.rows * s.heads * std::max(s.wk, s.wv) * sizeof(float)); }

size_t need_of(const Shape &s, bool backward) {
    const Cut c = cut_of(s.rows, s.num_seq, s.ptr != nullptr, s.heads, s.wk, s.wv);
    return enter_bytes(s, c) + gain_bytes(s, c) + (backward ? part_bytes(s, c) + share_bytes(s) : 0);
}

// rows of `heads` heads of `width` values, a distance ld from row to row and hd from head to head (0: one head for all, of inputs)
struct Heads {
    const void *at;
    int64_t ld, hd;
    int32_t heads, width;
    bool result;
};

// Elements of one row's heads may lie between those of another's (heads in front of rows); rows or heads of a result may not overlap
bool fits(const Heads &m, int64_t rows) {
    if (m.ld < 0 || m.hd < 0 || m.ld > CP_ATTENTION_MAX_DISTANCE || m.hd > CP_ATTENTION_MAX_HEAD_DISTANCE) return false;
    if (!m.result) return true;
    if (m.heads > 1 && m.hd < m.width) return false;
    if (rows > 1 && m.ld < m.width) return false;
    if (m.heads > 1 && rows > 1) {
        const bool inside = m.ld >= (m.heads - 1) * m.hd + m.width, outside = m.hd >= (rows - 1) * m.ld + m.width;
        return inside || outside;
    }
    return true;
}

// Where it lies: as equally distant rows where it can be put so, else all from its first element to its last
Extent extent(const Heads &m, int64_t rows, int type) {
    const int64_t each = (int64_t)type_bytes(type);
    if (!m.at || rows < 1) return {nullptr, 0, 0, 0, (size_t)each};
    const int64_t ld = rows > 1 ? m.ld : 0, hd = m.heads > 1 ? m.hd : 0;
    if (m.heads == 1 || hd == 0) return {m.at, ld ? rows : 1, m.width * each, (ld ? ld : m.width) * each, (size_t)each};
    if (rows == 1 || ld == 0) return {m.at, m.heads, m.width * each, hd * each, (size_t)each};
    if (hd == m.width && ld >= (int64_t)m.heads * hd) return {m.at, rows, m.heads * hd * each, ld * each, (size_t)each};
    if (ld == m.heads * hd) return {m.at, rows * m.heads, m.width * each, hd * each, (size_t)each};
    if (hd == rows * ld) return {m.at, rows * m.heads, m.width * each, ld * each, (size_t)each};
    const int64_t all = ((rows - 1) * ld + (m.heads - 1) * hd + m.width) * each;
    return {m.at, 1, all, all, (size_t)each};
}

// Whether two such share any byte: exactly where their rows are equally far apart, and their heads (slices of one buffer)
bool meet(const Heads &a, const Heads &b, int64_t rows, int type) {
    if (!a.at || !b.at || rows < 1) return false;
    const int64_t each = (int64_t)type_bytes(type);
    const bool alike = (rows == 1 || a.ld == b.ld) && (a.heads == 1 || b.heads == 1 || a.hd == b.hd);
    if (!alike || (rows > 1 && a.ld == 0)) return share(extent(a, rows, type), extent(b, rows, type));
    const int64_t ld = a.ld * each, hd = (a.heads > 1 ? a.hd : b.hd) * each, apart = (int64_t)(uintptr_t)b.at - (int64_t)(uintptr_t)a.at;
    const int64_t most = a.width * each - 1, least = 1 - b.width * each;      // how far behind one of a's heads one of b's may begin to touch it
    const auto upto = [&](int64_t off) { return off >= 0 ? off / ld : -((ld - 1 - off) / ld); };      // whole rows
    for (int64_t h = 1 - (int64_t)b.heads; h < a.heads; h++) {
        // one of b's heads lies `off` bytes behind one of a's in a row, and r rows on (a's rows may overlap) off + r ld
        const int64_t off = apart - h * hd;
        if (rows == 1 ? least <= off && off <= most : std::max(-upto(off - least), 1 - rows) <= std::min(upto(most - off), rows - 1)) return true;
    }
    return false;
}
// Whether a result shares memory with another result or with an input, rows of heads or others
bool in_the_way(std::initializer_list<Heads> in, std::initializer_list<Heads> out, std::initializer_list<Extent> more_in, std::initializer_list<Extent> more_out,
                int64_t rows, int type) {
    if (cpeval::in_the_way(more_in, more_out)) return true;
    for (const Heads *o = out.begin(); o != out.end(); o++) {
        for (const Heads &i : in)
            if (meet(i, *o, rows, type)) return true;
        for (const Heads *p = out.begin(); p != o; p++)
            if (meet(*p, *o, rows, type)) return true;
        if (cpeval::in_the_way(more_in, {extent(*o, rows, type)}) || cpeval::in_the_way(more_out, {extent(*o, rows, type)})) return true;
    }
    for (const Heads &i : in)
        if (cpeval::in_the_way({extent(i, rows, type)}, more_out)) return true;
    return false;
}

}  // namespace
}  // namespace attention
}  // namespace cpeval

using namespace cpeval;
using namespace cpeval::attention;

extern "C" {

int cp_linear_attention_workspace_bytes(int64_t rows, int32_t num_seq, int packed, int32_t heads, int32_t kv_heads, int32_t width_k,
                                        int32_t width_v, int backward, size_t *out_bytes) {
    if (!out_bytes) return CP_ERR_NULL;
    const int32_t some = 0;
    const Shape s{rows, num_seq, packed ? &some : nullptr, heads, kv_heads, width_k, width_v, CP_TYPE_F32};
    const int rc = check(s, 0);
    if (rc) return rc;
    *out_bytes = need_of(s, backward != 0);
    return CP_OK;
}

int cp_linear_attention_carry_states(int64_t rows, int32_t num_seq, int packed, int32_t heads, int32_t width_k, int32_t width_v, int64_t *out_states) {
    if (!out_states) return CP_ERR_NULL;
    const int32_t some = 0;
    const int rc = check({rows, num_seq, packed ? &some : nullptr, heads, heads, width_k, width_v, CP_TYPE_F32}, 0);
    if (rc) return rc;
    const Cut c = cut_of(rows, num_seq, packed != 0, heads, width_k, width_v);
    *out_states = c.split ? c.segments : 0;
    return CP_OK;
}

int cp_linear_attention(int64_t rows, int32_t num_seq, const int32_t *seq_ptr, int32_t heads, int32_t kv_heads, int32_t width_k,
                        int32_t width_v, int type, int reverse, const void *q, int64_t ldq, int64_t hdq, const void *k, int64_t ldk,
                        int64_t hdk, const void *v, int64_t ldv, int64_t hdv, const float *log_decay, float scale, const float *h0, void *o,
                        int64_t ldo, int64_t hdo, float *last, float *carry, void *workspace, size_t workspace_bytes, void *stream,
                        int32_t *status_out) {
    const Shape s{rows, num_seq, seq_ptr, heads, kv_heads, width_k, width_v, type};
    int rc = check(s, reverse);
    if (rc) return rc;
    if ((rows > 0 && (!q || !k || !v || !o)) || (seq_ptr && !status_out)) return CP_ERR_NULL;
    const Heads mq{q, ldq, hdq, heads, width_k, false}, mk{k, ldk, hdk, kv_heads, width_k, false}, mv{v, ldv, hdv, kv_heads, width_v, false},
        mo{o, ldo, hdo, heads, width_v, true};
    if (rows > 0 && (!fits(mq, rows) || !fits(mk, rows) || !fits(mv, rows) || !fits(mo, rows))) return CP_ERR_SIZE;
    const Cut c = cut_of(rows, num_seq, seq_ptr != nullptr, heads, width_k, width_v);
    const size_t enter = enter_bytes(s, c), need = gain_bytes(s, c) + (carry ? 0 : enter);
    if (need) {
        if (!workspace) return CP_ERR_NULL;
        if ((uintptr_t)workspace % kPolicyAlign || workspace_bytes < need) return CP_ERR_WORKSPACE;
    }
    const auto states = [&](const void *at) { return vector_at(at, (int64_t)num_seq * state_floats(s)); };
    if (attention::in_the_way({mq, mk, mv}, {mo}, {vector_at(log_decay, heads), states(h0), vector_at(seq_ptr, (int64_t)num_seq + 1, sizeof(int32_t))},
                              {states(last), vector_at(c.split ? carry : nullptr, c.segments * (int64_t)state_floats(s)),
                               vector_at(seq_ptr ? status_out : nullptr, 1, sizeof(int32_t)), vector_at(need ? workspace : nullptr, (int64_t)need, 1)},
                              rows, type))
        return CP_ERR_ARG;
    const hipStream_t st = (hipStream_t)stream;
    if (seq_ptr) hipLaunchKernelGGL(check_kernel, dim3(1), dim3(kThreads), 0, st, seq_ptr, num_seq, rows, status_out);
    if (last && (seq_ptr || rows == 0))
        hipLaunchKernelGGL(empty_kernel, dim3((unsigned)std::min(num_seq, 4096), 32), dim3(kThreads), 0, st, seq_ptr, rows / num_seq, num_seq,
                           (int64_t)state_floats(s), h0, last);
    if (rows == 0) return launched();
    Pass p{};
    p.rows = rows, p.len = rows / num_seq, p.ptr = seq_ptr, p.num_seq = num_seq;
    p.segments = c.segments, p.parts = c.parts, p.seg_rows = c.seg_rows;
    p.heads = heads, p.wa = width_k, p.wb = width_v, p.back = reverse != 0;
    p.s_in = 1.0f, p.s_out = scale, p.log_decay = log_decay;
    p.a = {q, ldq, hdq, 1}, p.b = {k, ldk, hdk, heads / kv_heads}, p.x = {v, ldv, hdv, heads / kv_heads};
    p.init = h0, p.last = last, p.o = o, p.ldo = ldo, p.hdo = hdo;
    if (c.split) {
        Gain *gain = (Gain *)workspace;
        float *at = carry ? carry : (float *)((char *)workspace + gain_bytes(s, c));
        rc = run_enter(type, p, at, gain, st);
        if (rc) return rc;
        p.enter = at;
    }
    return run(kOut, type, p, nullptr, nullptr, st);
}

int cp_linear_attention_backward(int64_t rows, int32_t num_seq, const int32_t *seq_ptr, int32_t heads, int32_t kv_heads, int32_t width_k,
                                 int32_t width_v, int type, int reverse, const void *d_o, int64_t lddo, int64_t hddo, const float *dlast,
                                 const void *q, int64_t ldq, int64_t hdq, const void *k, int64_t ldk, int64_t hdk, const void *v, int64_t ldv,
                                 int64_t hdv, const float *log_decay, float scale, const float *h0, const float *carry, void *dq, int64_t lddq,
                                 int64_t hddq, void *dk, int64_t lddk, int64_t hddk, void *dv, int64_t lddv, int64_t hddv, float *dlog_decay,
                                 float *dh0, void *workspace, size_t workspace_bytes, void *stream, int32_t *status_out) {
    const Shape s{rows, num_seq, seq_ptr, heads, kv_heads, width_k, width_v, type};
    int rc = check(s, reverse);
    if (rc) return rc;
    const Cut c = cut_of(rows, num_seq, seq_ptr != nullptr, heads, width_k, width_v);
    if ((rows > 0 && (!d_o || !q || !k || !v || !dq || !dk || !dv || (c.split && !carry))) || (seq_ptr && !status_out)) return CP_ERR_NULL;
    const Heads mo{d_o, lddo, hddo, heads, width_v, false}, mq{q, ldq, hdq, heads, width_k, false}, mk{k, ldk, hdk, kv_heads, width_k, false},
        mv{v, ldv, hdv, kv_heads, width_v, false}, nq{dq, lddq, hddq, heads, width_k, true}, nk{dk, lddk, hddk, kv_heads, width_k, true},
        nv{dv, lddv, hddv, kv_heads, width_v, true};
    if (rows > 0)
        for (const Heads *m : {&mo, &mq, &mk, &mv, &nq, &nk, &nv})
            if (!fits(*m, rows)) return CP_ERR_SIZE;
    const size_t need = need_of(s, true);
    if (rows > 0 || dlog_decay) {
        if (!workspace) return CP_ERR_NULL;
        if ((uintptr_t)workspace % kPolicyAlign || workspace_bytes < need) return CP_ERR_WORKSPACE;
    }
    const auto states = [&](const void *at) { return vector_at(at, (int64_t)num_seq * state_floats(s)); };
    const bool works = rows > 0 || dlog_decay;
    if (attention::in_the_way({mo, mq, mk, mv}, {nq, nk, nv},
                              {vector_at(log_decay, heads), states(h0), states(dlast), vector_at(c.split ? carry : nullptr, c.segments * (int64_t)state_floats(s)),
                               vector_at(seq_ptr, (int64_t)num_seq + 1, sizeof(int32_t))},
                              {vector_at(dlog_decay, heads), states(dh0), vector_at(seq_ptr ? status_out : nullptr, 1, sizeof(int32_t)),
                               vector_at(works ? workspace : nullptr, (int64_t)need, 1)},
                              rows, type))
        return CP_ERR_ARG;
    const hipStream_t st = (hipStream_t)stream;
    if (seq_ptr) hipLaunchKernelGGL(check_kernel, dim3(1), dim3(kThreads), 0, st, seq_ptr, num_seq, rows, status_out);
    if (dh0 && (seq_ptr || rows == 0))
        hipLaunchKernelGGL(empty_kernel, dim3((unsigned)std::min(num_seq, 4096), 32), dim3(kThreads), 0, st, seq_ptr, rows / num_seq, num_seq,
                           (int64_t)state_floats(s), dlast, dh0);
    char *room = (char *)workspace;
    Gain *gain = (Gain *)room;
    float *denter = (float *)(room + gain_bytes(s, c));
    double *part = (double *)(room + gain_bytes(s, c) + enter_bytes(s, c));
    float *share = (float *)((char *)part + part_bytes(s, c));
    const int32_t group = heads / kv_heads;
    if (rows == 0) {
        if (dlog_decay) hipLaunchKernelGGL(decay_kernel, dim3((unsigned)heads), dim3(kThreads), 0, st, part, (int64_t)0, dlog_decay);
        return launched();
    }
    const Operand in_do{d_o, lddo, hddo, 1}, in_q{q, ldq, hdq, 1}, in_k{k, ldk, hdk, group}, in_v{v, ldv, hdv, group};
    Pass p{};
    p.rows = rows, p.len = rows / num_seq, p.ptr = seq_ptr, p.num_seq = num_seq;
    p.segments = c.segments, p.parts = c.parts, p.seg_rows = c.seg_rows;
    p.heads = heads, p.log_decay = log_decay;

    // dv: keys read the gradient of the state
    Pass b = p;
    b.wa = width_k, b.wb = width_v, b.back = reverse == 0, b.last_first = true, b.shift = 1, b.s_in = scale, b.s_out = 1.0f;
    b.a = in_k, b.b = in_q, b.x = in_do, b.init = dlast, b.last = dh0;
    if (c.split) {
        rc = run_enter(type, b, denter, gain, st);
        if (rc) return rc;
        b.enter = denter;
    }
    // (heads that share keys and values: their gradients apart first, in 32 bits)
    const auto gradient = [&](Kind kind, Pass pass, void *to, int64_t ld, int64_t hd) {
        if (group == 1) {
            pass.o = to, pass.ldo = ld, pass.hdo = hd;
            return run(kind, type, pass, nullptr, nullptr, st);
        }
        pass.o = share, pass.hdo = pass.wb, pass.ldo = (int64_t)heads * pass.wb, pass.wide = true;
        const int code = run(kind, type, pass, nullptr, nullptr, st);
        if (code) return code;
        return by_type(type, [&](auto t) {
            using T = decltype(t);
            hipLaunchKernelGGL((pass.wb % 4 == 0 ? share_kernel<T, 4> : share_kernel<T, 1>), dim3((unsigned)std::min<int64_t>((rows + 3) / 4, 1 << 20)), dim3(kThreads), 0, st,
                               share, seq_ptr, num_seq, rows, heads, group, pass.wb, (T *)to, ld, hd);
            return launched();
        });
    };
    rc = gradient(kOut, b, dv, lddv, hddv);
    if (rc) return rc;
    // dk: values read it, transposed
    const int64_t parts = part_count(s, c);
    b.wa = width_v, b.wb = width_k, b.transposed = true, b.last = nullptr;
    b.a = in_v, b.b = in_do, b.x = in_q, b.d = in_k, b.part = part + parts / 2, b.part_step = parts;
    rc = gradient(dlog_decay ? kLeave : kOut, b, dk, lddk, hddk);
    if (rc) return rc;
    // dq: the gradients of the outputs read the state, transposed
    Pass a = p;
    a.wa = width_v, a.wb = width_k, a.transposed = true, a.back = reverse != 0, a.s_in = 1.0f, a.s_out = scale;
    a.a = in_do, a.b = in_v, a.x = in_k, a.d = in_q, a.init = h0, a.enter = c.split ? carry : nullptr;
    a.o = dq, a.ldo = lddq, a.hdo = hddq;
    a.dlast = dlast, a.denter = c.split ? denter : nullptr, a.part = part, a.part_step = parts;
    rc = run(dlog_decay ? kGrad : kOut, type, a, nullptr, nullptr, st);
    if (rc || !dlog_decay) return rc;
    hipLaunchKernelGGL(decay_kernel, dim3((unsigned)heads), dim3(kThreads), 0, st, part, parts, dlog_decay);
    return launched();
}

int cp_linear_attention_step(int32_t num_seq, int32_t heads, int32_t kv_heads, int32_t width_k, int32_t width_v, int type, const void *q,
                             int64_t ldq, int64_t hdq, const void *k, int64_t ldk, int64_t hdk, const void *v, int64_t ldv, int64_t hdv,
                             const float *log_decay, float scale, float *state, int32_t num_slots, const int32_t *slots, void *o, int64_t ldo,
                             int64_t hdo, void *stream, int32_t *status_out) {
    if (!known_type(type)) return CP_ERR_ARG;
    if (num_seq < 0 || num_slots < 1 || (!slots && num_seq > num_slots)) return CP_ERR_SIZE;
    const Shape s{num_seq, 1, nullptr, heads, kv_heads, width_k, width_v, type};
    const int rc = check(s, 0);
    if (rc) return rc;
    if ((int64_t)num_seq * heads > INT32_MAX) return CP_ERR_SIZE;
    if ((num_seq > 0 && (!q || !k || !v || !o)) || !state || (slots && !status_out)) return CP_ERR_NULL;
    const Heads mq{q, ldq, hdq, heads, width_k, false}, mk{k, ldk, hdk, kv_heads, width_k, false}, mv{v, ldv, hdv, kv_heads, width_v, false},
        mo{o, ldo, hdo, heads, width_v, true};
    if (num_seq > 0 && (!fits(mq, num_seq) || !fits(mk, num_seq) || !fits(mv, num_seq) || !fits(mo, num_seq))) return CP_ERR_SIZE;
    if (attention::in_the_way({mq, mk, mv}, {mo}, {vector_at(log_decay, heads), vector_at(slots, num_seq, sizeof(int32_t))},
                              {vector_at(state, (int64_t)num_slots * state_floats(s)), vector_at(slots ? status_out : nullptr, 1, sizeof(int32_t))}, num_seq, type))
        return CP_ERR_ARG;
    const hipStream_t st = (hipStream_t)stream;
    if (slots) hipLaunchKernelGGL(set_status_kernel, dim3(1), dim3(1), 0, st, status_out, CP_STATUS_OK);
    if (num_seq == 0) return launched();
    const Step p{num_seq, heads, width_k, width_v, num_slots, {q, ldq, hdq, 1}, {k, ldk, hdk, heads / kv_heads}, {v, ldv, hdv, heads / kv_heads},
                 log_decay, scale, state, slots, o, ldo, hdo, status_out};
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL((width_v % 4 == 0 ? step_kernel<T, 4> : step_kernel<T, 1>), grid_of((int64_t)num_seq * heads), dim3(kThreads), 0, st, p);
        return launched();
    });
}

}  // extern "C"
