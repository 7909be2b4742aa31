// Log probabilities of given classes with the entropy and the best alternatives of each row (bmgd_log_probs), and their gradient
// (bmgd_log_probs_backward).
//
//     M = max_c z_c,  s = sum_c e^(z_c - M),  t = sum_c (z_c - M) e^(z_c - M)
//     log p_c = (z_c - M) - log s,   entropy H = log s - t / s
//     gradient of  a log p_y + b H:   dz_c = a ([c = y] - p_c) - b p_c (log p_c + H)
//     alternatives: the K largest logits in falling order, equal ones by rising class
//
// One pass over the row keeps a running maximum with both sums in every thread; t needs no second pass because both sums are
// carried to a larger maximum together: s' = s f, t' = (t + s (M - M')) f with f = e^(M - M').  While a thread reads, its sums may stay with
// an earlier maximum as long as the present one is no more than 40 above it (no term overflows): among 32 lanes some maximum rises in nearly every round.
// The sums are taken in powers of two, 2^(z L - m) with L = log2 e in fp32 and m = M L rounded: one multiply-add a logit.  What m is
// rounded by is the same in every term; it is put right once, in log s (row_score).
//
// Alternatives.  The maxima of 32 parts of the row (the threads of equal lane) bound the K-th
// largest logit from below: at least K of the parts hold a logit at or above the K-th largest of them.  While it reads, a thread leaves the
// maximum of each of its stretches in shared memory; only stretches that reach the bound are looked at again (a few dozen of a row of independent logits, from L2), what reaches the
// bound is put aside, and its K largest are ranked by counting.  Rows with more candidates than there is room are taken value by value: largest below the last one, with all that equal it.
// These are rows of thousands of equal logits, or with a mask that leaves fewer than K; rows of 161 to 255 classes in 16-bit types with K above C / 8 (fewer than K of the parts have a logit,
// so nothing is ruled out); and with K near 32 ordinary ones too: at the lowest of 32 maxima some 130 independent logits are left on average, and often more than 160 (16384 x 4000 with
// 20 alternatives 78 us, with 32 780; 8191 x 200 16 and 95).
//
// A row with NaN or +Inf has NaN for its log probability and entropy; in the order of the alternatives NaN is largest.  A row whose logits are
// all -Inf has no distribution: log probability and entropy 0, no gradient, alternatives -Inf from class 0 on.
//
// What bounds it: the exponentials (four lanes of a quarter SM a clock) and memory, about equally in 16-bit types.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>
#include <type_traits>

#include "values.cuh"

namespace bmgdk {

constexpr int kMostAlternatives = 32;
constexpr float kFarBelow = -200.f;  // e^-200 is 0 in fp32, as kFar2

struct LogProbParams {
    const void* z;
    const int* y;               // null: no labels
    float *logprob, *entropy;   // null: not wanted
    float* saved;               // [rows][3]: M, log s, H
    int* index;                 // [rows][top]
    float* value;
    const float *dlogprob, *dentropy;  // backward; null: zeros
    void* dz;
    long long ld, ld_dz, rows;
    int C, top, far;            // far: dz is not to stay in L2
};

// Maximum M (NaN wins), its stand-in m = M L, and sums of 2^(z L - m) and (z L - m) 2^(z L - m).  |M| is at most kWide where the sums
// are used (a row beyond is done anew by score_careful); m is held within it, which leaves the sums of what is smaller zero.
struct Score {
    float m, s, t;
};
constexpr float kWide = 16777216.f;     // 2^24: m is M L within one
constexpr float kFar2 = -300.f;         // 2^-300 is 0 in fp32: a logit that far below (-Inf too) counts for nothing, and 0 times it is 0
__device__ __forceinline__ float score_max(float a, float b) {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
// (rounded by itself: within a multiply-add the product would be another number, and carrying sums on to the same maximum no longer one)
__device__ __forceinline__ float score_base(float m) { return __fmul_rn(fminf(fmaxf(m, -kWide), kWide), kLog2e); }
__device__ __forceinline__ float power_of_two(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ void score_raise(Score& a, float m) {  // to a maximum not below its own
    const float d = fmaxf(score_base(a.m) - score_base(m), kFar2), f = power_of_two(d);  // (a.m = -Inf: both sums are 0)
    a.t = fmaf(a.s, d, a.t) * f;
    a.s *= f;
    a.m = m;
}
__device__ __forceinline__ Score score_warp(Score a) {
    float m;
    asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(a.m));
    score_raise(a, m);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a.s += __shfl_xor_sync(0xFFFFFFFFu, a.s, o);
        a.t += __shfl_xor_sync(0xFFFFFFFFu, a.t, o);
    }
    return a;
}
template <typename T>
__device__ __forceinline__ float score_piece_max(const uint4& w) {
    if constexpr (sizeof(T) == 4) {
        float x[4];
        unpack_piece<T>(w, x);
        return score_max(score_max(x[0], x[1]), score_max(x[2], x[3]));
    } else if constexpr (std::is_same<T, __half>::value) {
        const __half2* p = reinterpret_cast<const __half2*>(&w);
        const float2 m = __half22float2(__hmax2_nan(__hmax2_nan(p[0], p[1]), __hmax2_nan(p[2], p[3])));
        return score_max(m.x, m.y);
    } else {
        const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&w);
        const float2 m = __bfloat1622float2(__hmax2_nan(__hmax2_nan(p[0], p[1]), __hmax2_nan(p[2], p[3])));
        return score_max(m.x, m.y);
    }
}
// Whether a row's maximum asks for the careful form
__device__ __forceinline__ bool score_wide(float m) { return fabsf(m) < INFINITY && fabsf(m) > kWide; }
// adds a piece to sums against a base.  (Raising what is far below in its 16-bit form, two at a time, took longer: 8191 x 50257 155 us
// instead of 151.)
template <typename T>
__device__ __forceinline__ void score_piece(const uint4& w, float base, float& s, float& t) {
    constexpr int VE = Piece<T>::kValues;
    float x[VE];
    unpack_piece<T>(w, x);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        const float d = fmaxf(fmaf(x[e], kLog2e, -base), kFar2), p = power_of_two(d);
        s += p;
        t = fmaf(d, p, t);
    }
}
// largest value of four pieces
template <typename T>
__device__ __forceinline__ float score_pieces_max(const uint4 (&w)[4]) {
    if constexpr (sizeof(T) == 4) {
        return score_max(score_max(score_piece_max<T>(w[0]), score_piece_max<T>(w[1])), score_max(score_piece_max<T>(w[2]), score_piece_max<T>(w[3])));
    } else {
        typedef typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type Two;
        const Two *a = reinterpret_cast<const Two*>(&w[0]), *b = reinterpret_cast<const Two*>(&w[1]), *c = reinterpret_cast<const Two*>(&w[2]), *d = reinterpret_cast<const Two*>(&w[3]);
        uint4 m;
        Two* t = reinterpret_cast<Two*>(&m);
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = __hmax2_nan(__hmax2_nan(a[i], b[i]), __hmax2_nan(c[i], d[i]));
        return score_piece_max<T>(m);
    }
}
// A thread's sums while it reads: against `from`, the largest value at the time they were last carried on.
template <typename T>
struct Reading {
    Score a{-INFINITY, 0.f, 0.f};  // (a.m: the largest value so far)
    float from = -INFINITY, base = 0.f;
    __device__ __forceinline__ void reach(float m) {
        a.m = score_max(a.m, m);
        if (!(a.m - from <= 40.f)) {  // (also the first time, and while all is -Inf)
            Score b{from, a.s, a.t};
            score_raise(b, a.m);
            a = b;
            from = a.m;
            base = score_base(from);
        }
    }
    __device__ __forceinline__ float add_four(const uint4 (&w)[4]) {  // returns the largest of them
        const float m = score_pieces_max<T>(w);
        reach(m);
        float s = 0.f, t = 0.f;  // (two sums each: the additions follow one another)
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
            score_piece<T>(w[k], base, a.s, a.t);
            score_piece<T>(w[k + 1], base, s, t);
        }
        a.s += s;
        a.t += t;
        return m;
    }
    __device__ __forceinline__ void add_one(float x) {
        reach(x);
        const float d = fmaxf(fmaf(x, kLog2e, -base), kFar2), p = power_of_two(d);
        a.s += p;
        a.t = fmaf(d, p, a.t);
    }
    __device__ __forceinline__ Score done() const {
        Score b{from, a.s, a.t};
        score_raise(b, a.m);
        return b;
    }
};
// What a row's sums say.
struct RowScore {
    float m, log_s, entropy;  // log p = (z - m) - log_s
    bool nothing, broken;     // no distribution; NaN or +Inf
};
__device__ __forceinline__ RowScore row_score(const Score& a) {
    RowScore r;
    r.m = a.m;
    r.nothing = a.m == -INFINITY;
    r.broken = !(a.m < INFINITY);
    const float nan = __uint_as_float(0x7FC00000u), ln2 = 0.69314718056f;
    const float log_s = logf(a.s);
    r.entropy = r.broken ? nan : r.nothing ? 0.f : log_s - ln2 * (a.t / a.s);
    r.log_s = r.broken ? nan : r.nothing ? 0.f : log_s - ln2 * fmaf(a.m, kLog2e, -score_base(a.m));
    return r;
}

// ---- order of the alternatives: 32 bits that rise with the value (-0 as 0, NaN above all), and back
__device__ __forceinline__ uint32_t rank_bits(float x) {
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float rank_value(uint32_t r) {
    if (r == 0xFFFFFFFFu) return __uint_as_float(0x7FC00000u);
    return __uint_as_float(r & 0x80000000u ? r & 0x7FFFFFFFu : ~r);
}
__device__ __forceinline__ unsigned long long candidate(uint32_t rank, int c) { return (unsigned long long)rank << 32 | (0xFFFFFFFFu - (uint32_t)c); }

// What the threads of a row share (TH = 32: those of a warp).
template <int TH, int ROOM>
struct LogProbShared {
    Score part[TH / 32];
    RowScore row;
    float lanes[TH / 32][32];
    unsigned long long found[ROOM];
    int spots[ROOM], classes[ROOM];
    int spot_count, found_count;
    uint32_t bound;
    uint32_t best[TH / 32], place[TH / 32], equal[TH / 32];
};
template <int TH>
__device__ __forceinline__ void row_sync() {
    if constexpr (TH == 32) __syncwarp();
    else __syncthreads();
}

// The K largest taken value by value, for rows with many candidates.  All threads of the row call it; found holds them in order.
template <typename T, int TH, int ROOM>
__device__ __noinline__ void take_by_value(const T* z, int C, int top, LogProbShared<TH, ROOM>& S) {
    const int tid = TH == 32 ? (int)threadIdx.x & 31 : (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int have = 0;
    bool any_limit = false;
    uint32_t limit = 0;
    while (have < top) {
        // largest value below the limit, where it first stands, how often it occurs
        uint32_t best = 0, place = 0xFFFFFFFFu, equal = 0;
        for (int c = tid; c < C; c += TH) {
            const uint32_t r = rank_bits(to_f32(z[c]));
            if (any_limit && r >= limit) continue;
            if (equal == 0 || r > best) { best = r; place = (uint32_t)c; equal = 1; }
            else if (r == best) ++equal;
        }
        uint32_t b = __reduce_max_sync(0xFFFFFFFFu, equal ? best : 0u);
        uint32_t p = __reduce_min_sync(0xFFFFFFFFu, equal && best == b ? place : 0xFFFFFFFFu);
        uint32_t n = __reduce_add_sync(0xFFFFFFFFu, equal && best == b ? equal : 0u);
        if constexpr (TH > 32) {
            if (lane == 0) { S.best[warp] = b; S.place[warp] = p; S.equal[warp] = n; }
            __syncthreads();
            b = 0;
            for (int k = 0; k < TH / 32; ++k)
                if (S.equal[k] != 0) b = max(b, S.best[k]);
            p = 0xFFFFFFFFu;
            n = 0;
            for (int k = 0; k < TH / 32; ++k)
                if (S.equal[k] != 0 && S.best[k] == b) { p = min(p, S.place[k]); n += S.equal[k]; }
            __syncthreads();
        }
        if (n == 0) break;  // (top <= C: does not happen)
        const int want = min((int)n, top - have);
        if (want == 1) {
            if (tid == 0) S.found[have] = candidate(b, (int)p);
        } else {  // in the order of the classes, from the first on
            int got = 0;
            for (int c0 = (int)p; c0 < C && got < want; c0 += TH) {
                const int c = c0 + tid;
                const bool is = c < C && rank_bits(to_f32(z[c])) == b;
                const uint32_t mask = __ballot_sync(0xFFFFFFFFu, is);
                int before = __popc(mask & ((1u << lane) - 1u)), all = __popc(mask);
                if constexpr (TH > 32) {
                    if (lane == 0) S.equal[warp] = (uint32_t)all;
                    __syncthreads();
                    all = 0;
                    for (int k = 0; k < TH / 32; ++k) {
                        if (k == warp) before += all;
                        all += (int)S.equal[k];
                    }
                    __syncthreads();
                }
                if (is && got + before < want) S.found[have + got + before] = candidate(b, c);
                got += all;
            }
        }
        have += want;
        limit = b;
        any_limit = true;
    }
    row_sync<TH>();
}

// A row whose maximum is beyond +-2^24 (all logits at a type's lowest value, say), against differences that are taken first: all
// threads of the row call it, with its maximum; each returns the whole row's sums, as row_score gives them.
template <typename T, int TH, int ROOM>
__device__ __noinline__ RowScore score_careful(const T* z, int C, float m, LogProbShared<TH, ROOM>& S) {
    const int tid = TH == 32 ? (int)threadIdx.x & 31 : (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    float s = 0.f, t = 0.f;
    for (int c = tid; c < C; c += TH) {
        const float d = fmaxf(to_f32(z[c]) - m, kFarBelow), p = exp_fast(d);
        s += p;
        t = fmaf(d, p, t);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
    }
    if constexpr (TH > 32) {
        __syncthreads();  // (the sums before these have been read)
        if (lane == 0) S.part[warp] = Score{m, s, t};
        __syncthreads();
        s = t = 0.f;
        for (int k = 0; k < TH / 32; ++k) {
            s += S.part[k].s;
            t += S.part[k].t;
        }
    }
    const float log_s = logf(s);
    return RowScore{m, log_s, log_s - t / s, false, false};
}

// TH threads to a row (TH = 32: a warp, eight rows to a block), rows taken with the grid's stride: the first pieces of the next row are
// fetched before this one's sums are joined.  Small blocks with many registers: 8191 x 50257 bf16 took 135 us with 64 threads and 85 registers (by now 132 with 80), 142
// with 128, 157 with 256; 142 with 64 threads and 64 registers.
template <typename T, int TH, bool TOP>
__global__ void __launch_bounds__(TH == 32 ? 256 : TH, TH == 32 ? 3 : TH >= 512 ? 1 : 768 / TH) logprob_kernel(const __grid_constant__ LogProbParams P) {
    constexpr int VE = Piece<T>::kValues, kAhead = 4, kWarps = TH / 32, kRound = kAhead * TH;
    constexpr int kRoom = 160;
    // maxima kept of a row's stretches, each thread its own; as few bytes as will do, because the loads under way need the rest for L1 (12 blocks to an
    // SM of 17 KB each: 8191 x 50257 with 20 alternatives 209 us, of 8 KB 173)
    constexpr int kStretches = 4096 / (int)sizeof(T);
    // (two sets that take turns: a thread that begins a row may meet others that still read what they share of the row before)
    __shared__ LogProbShared<TH, TOP ? kRoom : 1> shared[TH == 32 ? 8 : 1][TH == 32 ? 1 : 2];
    __shared__ T stretch[TOP && TH > 32 ? kStretches : 1];
    const int tid = TH == 32 ? (int)threadIdx.x & 31 : (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long step = TH == 32 ? gridDim.x * 8ll : (long long)gridDim.x;
    uint4 next[kAhead];
    float edge = -INFINITY;
    auto begin = [&](long long i) {  // the first pieces of a row
        const T* z = static_cast<const T*>(P.z) + i * P.ld;
        const RowPieces<T> row(z, P.C);
        const uint4* src = reinterpret_cast<const uint4*>(z + row.head);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (tid + k * TH < row.pieces) next[k] = src[tid + k * TH];
        if (tid < row.edges) edge = to_f32(z[row.edge(tid)]);
    };
    long long i = TH == 32 ? blockIdx.x * 8ll + (threadIdx.x >> 5) : (long long)blockIdx.x;
    if (i < P.rows) begin(i);
    for (int turn = 0; i < P.rows; i += step, turn ^= 1) {
        auto& S = shared[TH == 32 ? threadIdx.x >> 5 : 0][TH == 32 ? 0 : turn];
        const T* z = static_cast<const T*>(P.z) + i * P.ld;
        const RowPieces<T> row(z, P.C);
        const uint4* src = reinterpret_cast<const uint4*>(z + row.head);
        const int pieces = row.pieces;
        const int label = P.y ? __ldg(P.y + i) : -1;
        float at_label = 0.f;
        if (tid == 0 && label >= 0 && label < P.C) at_label = to_f32(z[label]);

        // ---- one pass: the sums of each thread, and its maximum
        Reading<T> read;
        const bool odd = tid < row.edges;
        const float edge_value = edge;
        if (odd) read.add_one(edge_value);
        uint4 w[kAhead];
        // rounds in which every thread has kAhead pieces, two to a turn: one set of registers is filled while the other is worked on
        const int rounds = pieces / kRound;
        const int span = (rounds + kStretches / TH - 1) / (kStretches / TH);  // rounds of a stretch
        int stretches = 0, in_stretch = 0;
        float highest = -INFINITY;
        auto add = [&](const uint4 (&v)[kAhead]) {
            const float m = read.add_four(v);
            if constexpr (TOP && TH > 32) {
                highest = score_max(highest, m);
                if (++in_stretch == span) {
                    stretch[stretches++ * TH + tid] = from_f32<T>(highest);  // (exact: it is one of them)
                    highest = -INFINITY;
                    in_stretch = 0;
                }
            }
        };
        const uint4* at = src + tid;
        int left = rounds;
        for (; left > 2; left -= 2, at += 2 * kRound) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) w[k] = at[kRound + k * TH];
            add(next);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) next[k] = at[2 * kRound + k * TH];
            add(w);
        }
        int k0 = tid + (rounds - left) * kRound;
        for (; left > 0; --left) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (k0 + (kAhead + k) * TH < pieces) w[k] = src[k0 + (kAhead + k) * TH];
            add(next);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) next[k] = w[k];
            k0 += kRound;
        }
        if (TOP && TH > 32 && in_stretch > 0) stretch[stretches++ * TH + tid] = from_f32<T>(highest);  // (exact: it is one of them)
        // what is left of the row, up to kAhead pieces a thread: they stay in registers
        highest = -INFINITY;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            w[k] = next[k];
            if (k0 + k * TH < pieces) highest = score_max(highest, score_piece_max<T>(w[k]));
        }
        read.reach(highest);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (k0 + k * TH < pieces) score_piece<T>(w[k], read.base, read.a.s, read.a.t);
        Score a = read.done();
        if (i + step < P.rows) begin(i + step);
        const float own = a.m;  // this thread's maximum
        if constexpr (TOP && TH > 32) S.lanes[warp][lane] = own;
        a = score_warp(a);
        if constexpr (TH > 32) {
            if (lane == 0) S.part[warp] = a;
        }
        if constexpr (TOP) {
            if (tid == 0) S.spot_count = S.found_count = 0;
        }
        row_sync<TH>();
        // the row's sums and, for the alternatives, the bound: by one warp
        RowScore r{};
        uint32_t g = 0;
        if (TH == 32 || warp == 0) {
            if constexpr (TH > 32) a = score_warp(lane < kWarps ? S.part[lane] : Score{-INFINITY, 0.f, 0.f});
            r = row_score(a);
        }
        if constexpr (TH > 32) {
            if (warp == 0 && lane == 0) S.row = r;
        }
        if constexpr (TOP) {
            if (TH == 32 || warp == 0) {
                g = rank_bits(own);
                if constexpr (TH > 32) {
                    float m = S.lanes[0][lane];
#pragma unroll
                    for (int k = 1; k < kWarps; ++k) m = score_max(m, S.lanes[k][lane]);
                    g = rank_bits(m);
                }
                // the 32 parts' maxima in falling order, lane by lane
#pragma unroll
                for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
                    for (int j = k >> 1; j > 0; j >>= 1) {
                        const uint32_t o = __shfl_xor_sync(0xFFFFFFFFu, g, j);
                        g = ((lane & k) == 0) == ((lane & j) == 0) ? max(g, o) : min(g, o);
                    }
                g = __shfl_sync(0xFFFFFFFFu, g, P.top - 1);
                if (TH > 32 && lane == 0) S.bound = g;
            }
        }
        bool wide = TH == 32 && score_wide(r.m);
        if constexpr (TH > 32 && TOP) {
            __syncthreads();
            r = S.row;
            g = S.bound;
            wide = score_wide(r.m);
        }
        if constexpr (TH > 32 && !TOP) {  // (no other barrier is needed: whether the row is one of the rare ones, each thread sees for itself)
            float m = S.part[0].m;
#pragma unroll
            for (int k = 1; k < kWarps; ++k) m = score_max(m, S.part[k].m);
            wide = score_wide(m);
            if (wide) r.m = m;
        }
        if (wide) r = score_careful<T>(z, P.C, r.m, S);
        const float nan = __uint_as_float(0x7FC00000u);
        if (tid == 0) {
            if (P.logprob) P.logprob[i] = label < 0 || label >= P.C || r.nothing ? 0.f : (at_label - r.m) - r.log_s;
            if (P.entropy) P.entropy[i] = r.entropy;
            if (P.saved) {
                P.saved[3 * i] = r.m;
                P.saved[3 * i + 1] = r.log_s;
                P.saved[3 * i + 2] = r.entropy;
            }
        }
        if constexpr (TOP) {
            // ---- the alternatives
            const int top = P.top;
            const float bound = rank_value(g);
            auto found_one = [&](int c) {
                const int n = atomicAdd(&S.found_count, 1);
                if (n < kRoom) S.classes[n] = c;
            };
            auto consider_piece = [&](const uint4& v, int p) {
                if (score_piece_max<T>(v) < bound) return;  // (NaN is no less)
                float x[VE];
                unpack_piece<T>(v, x);
                uint32_t hits = 0;
#pragma unroll
                for (int e = 0; e < VE; ++e) hits |= x[e] < bound ? 0u : 1u << e;
                for (; hits; hits &= hits - 1) found_one(row.column(p) + __ffs(hits) - 1);
            };
            if (odd && !(edge_value < bound)) found_one(row.edge(tid));
            if (!(highest < bound)) {
#pragma unroll
                for (int k = 0; k < kAhead; ++k)
                    if (k0 + k * TH < pieces) consider_piece(w[k], k0 + k * TH);
            }
            if (rounds > 0) {
                if constexpr (TH > 32) {
#pragma unroll 4
                    for (int k = 0; k < stretches; ++k)
                        if (!(to_f32(stretch[k * TH + tid]) < bound)) {
                            const int n = atomicAdd(&S.spot_count, 1);
                            if (n < kRoom) S.spots[n] = k * TH + tid;
                        }
                    __syncthreads();
                    // all threads look at the pieces of the stretches found: `reach` pieces each, TH apart
                    const unsigned reach = (unsigned)span * kAhead, items = (unsigned)min(S.spot_count, kRoom) * reach;
#pragma unroll 2
                    for (unsigned k = tid; k < items; k += TH) {
                        const unsigned o = k / reach, spot = (unsigned)S.spots[o], first = spot / TH * reach;
                        const unsigned p = (first + (k - o * reach)) * TH + spot % TH;
                        if (p < (unsigned)(rounds * kRound)) consider_piece(src[p], (int)p);
                    }
                } else {  // (a warp's row of one round: its pieces are read again)
                    for (int p = tid; p < rounds * kRound; p += TH) consider_piece(src[p], p);
                }
            }
            row_sync<TH>();
            int found = max(S.found_count, S.spot_count);
            if (found > kRoom) {
                row_sync<TH>();
                take_by_value<T>(z, P.C, top, S);
                found = top;
            } else {
                found = S.found_count;
                for (int k = tid; k < found; k += TH) S.found[k] = candidate(rank_bits(to_f32(z[S.classes[k]])), S.classes[k]);
                row_sync<TH>();
            }
            for (int k = tid; k < found; k += TH) {
                const unsigned long long mine = S.found[k];
                int rank = 0;
#pragma unroll 4
                for (int j = 0; j < found; ++j) rank += S.found[j] > mine ? 1 : 0;
                if (rank >= top) continue;
                const float x = rank_value((uint32_t)(mine >> 32));
                P.index[i * top + rank] = (int)(0xFFFFFFFFu - (uint32_t)mine);
                P.value[i * top + rank] = r.broken ? nan : r.nothing ? -INFINITY : (x - r.m) - r.log_s;
            }
            if constexpr (TH == 32) __syncwarp();  // (a warp has one set)
        }
    }
}

// ---- gradient: each logit read once, its gradient written once.  gridDim.y blocks share a row.
template <typename T, int TH>
__global__ void __launch_bounds__(TH == 32 ? 256 : TH) logprob_back_kernel(const __grid_constant__ LogProbParams P) {
    constexpr int VE = Piece<T>::kValues, kAhead = 4;
    const int tid = TH == 32 ? (int)threadIdx.x & 31 : (int)threadIdx.x;
    const long long i = TH == 32 ? blockIdx.x * 8ll + (threadIdx.x >> 5) : (long long)blockIdx.x;
    if (i >= P.rows) return;
    const T* z = static_cast<const T*>(P.z) + i * P.ld;
    T* dz = static_cast<T*>(P.dz) + i * P.ld_dz;
    const RowPieces<T> row(z, P.C);
    const int label = P.y ? P.y[i] : -1;
    const float m = P.saved[3 * i], log_s = P.saved[3 * i + 1], entropy = P.saved[3 * i + 2];
    const bool labelled_row = P.dlogprob && label >= 0 && label < P.C;
    const bool nothing = m == -INFINITY || !(labelled_row || P.dentropy);  // no distribution, or nothing asked of it
    const float a = labelled_row && !nothing ? P.dlogprob[i] : 0.f, b = P.dentropy && !nothing ? P.dentropy[i] : 0.f;
    // dz = p (k0 + k1 log p), and a for the label
    const float k0 = -(a + b * entropy), k1 = -b, base = m;
    auto one = [&](float x, int c) {
        const float lp = fmaxf((x - base) - log_s, kFarBelow), v = exp_fast(lp) * (k0 + k1 * lp);
        return c == label ? v + a : v;
    };
    if (!nothing && blockIdx.y == 0 && tid < row.edges) dz[row.edge(tid)] = from_f32<T>(one(to_f32(z[row.edge(tid)]), row.edge(tid)));
    if (nothing) {  // (zeros, whatever the row holds)
        for (int c = (int)blockIdx.y * TH + tid; c < P.C; c += (int)gridDim.y * TH) dz[c] = from_f32<T>(0.f);
        return;
    }
    const Pair minus_m(-base), minus_s(-log_s), log2e(kLog2e), p0(k0), p1(k1);
    for (int q0 = (int)blockIdx.y * kAhead * TH + tid; q0 < row.pieces; q0 += (int)gridDim.y * kAhead * TH) {
        uint4 w[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (q0 + k * TH < row.pieces) w[k] = load_piece(z + row.column(q0 + k * TH));
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (q0 + k * TH >= row.pieces) continue;
            const int c = row.column(q0 + k * TH);
            float x[VE];
            unpack_piece<T>(w[k], x);
            uint4 out;
            T* t = reinterpret_cast<T*>(&out);
            const bool labelled = label >= c && label < c + VE;
#pragma unroll
            for (int e = 0; e < VE; e += 2) {
                float2 d = (Pair(x[e], x[e + 1]) + minus_m + minus_s).both();
                d.x = fmaxf(d.x, kFarBelow);
                d.y = fmaxf(d.y, kFarBelow);
                const Pair dd(d.x, d.y);
                float2 p = (dd * log2e).both();
                asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(p.x));
                asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(p.y));
                float2 v = (Pair(p.x, p.y) * multiply_add(dd, p1, p0)).both();
                if (labelled) {
                    if (c + e == label) v.x += a;
                    if (c + e + 1 == label) v.y += a;
                }
                put_pair<T>(t + e, Pair(v.x, v.y));
            }
            store_piece(dz + c, out, P.far != 0);
        }
    }
}

}  // namespace bmgdk
