// Log probabilities of given classes with the entropy and the best alternatives of each row (bmgd_log_probs), and their gradient
// (bmgd_log_probs_backward).
//
//     M = max_c z_c,  s = sum_c e^(z_c - M),  t = sum_c (z_c - M) e^(z_c - M)
//     log p_c = (z_c - M) - log s,   entropy H = log s - t / s
//     gradient of  a log p_y + b H:   dz_c = a ([c = y] - p_c) - b p_c (log p_c + H)
//     alternatives: the K largest logits in falling order, equal ones by rising class
//
// One pass over the row keeps a running maximum with both sums in every thread; t needs no second pass because both sums are
// carried to a larger maximum together: s' = s f, t' = (t + s (M - M')) f with f = e^(M - M').
//
// Alternatives.  Each thread's maximum is known after that pass.  The maxima of 32 parts of the row (the threads of equal lane) bound the K-th
// largest logit from below: at least K of the parts hold a logit at or above the K-th largest of them.  Only threads whose own
// maximum reaches that bound look at their logits again (a few dozen of a row of independent logits, from L2), what reaches the
// bound is put aside, and its K largest are ranked by counting.  Rows with more candidates than there is room (thousands of equal logits, a mask that
// leaves fewer than K) are taken value by value: largest below the last one, with all that equal it.
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
constexpr float kFarBelow = -200.f;  // e^-200 is 0 in fp32: a logit that far below (-Inf too) counts for nothing, and 0 times it is 0

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
    int C, top;
};

// Maximum (NaN wins), sum of exponentials and of exponentials times their distance from it.
struct Score {
    float m, s, t;
};
__device__ __forceinline__ float score_base(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float score_max(float a, float b) {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
__device__ __forceinline__ void score_raise(Score& a, float m) {  // to a maximum not below its own
    const float d = fmaxf(a.m - score_base(m), kFarBelow), f = exp_fast(d);  // (a.m = -Inf: both sums are 0)
    a.t = (a.t + a.s * d) * f;
    a.s *= f;
    a.m = m;
}
__device__ __forceinline__ Score score_join(Score a, Score b) {
    const float m = score_max(a.m, b.m);
    score_raise(a, m);
    score_raise(b, m);
    return Score{m, a.s + b.s, a.t + b.t};
}
__device__ __forceinline__ Score score_lanes(Score a) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        a = score_join(a, Score{__shfl_xor_sync(0xFFFFFFFFu, a.m, o), __shfl_xor_sync(0xFFFFFFFFu, a.s, o), __shfl_xor_sync(0xFFFFFFFFu, a.t, o)});
    return a;
}
__device__ __forceinline__ void score_one(Score& a, float x) {
    const float m = score_max(a.m, x);
    if (!(m <= a.m)) score_raise(a, m);
    const float d = fmaxf(x - score_base(a.m), kFarBelow), p = exp_fast(d);
    a.s += p;
    a.t += d * p;
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
// adds a piece to sums relative to the present maximum
template <typename T>
__device__ __forceinline__ void score_piece(const uint4& w, const Pair& minus_m, Pair& s, Pair& t) {
    constexpr int VE = Piece<T>::kValues;
    const Pair log2e(kLog2e);
    float x[VE];
    unpack_piece<T>(w, x);
#pragma unroll
    for (int e = 0; e < VE; e += 2) {
        float2 d = (Pair(x[e], x[e + 1]) + minus_m).both();
        d.x = fmaxf(d.x, kFarBelow);
        d.y = fmaxf(d.y, kFarBelow);
        const Pair dd(d.x, d.y);
        float2 p = (dd * log2e).both();
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(p.x));
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(p.y));
        const Pair pp(p.x, p.y);
        s = s + pp;
        t = multiply_add(dd, pp, t);
    }
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
    float lanes[TH / 32][32];
    int owners[TH];
    unsigned long long found[ROOM];
    int owner_count, found_count;
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

// TH threads to a row (TH = 32: a warp, eight rows to a block).
template <typename T, int TH, bool TOP>
__global__ void __launch_bounds__(TH == 32 ? 256 : TH, TH == 32 ? 4 : TH >= 512 ? 2 : 1024 / TH) logprob_kernel(const __grid_constant__ LogProbParams P) {
    constexpr int VE = Piece<T>::kValues, kAhead = 4, kWarps = TH / 32;
    constexpr int kRoom = TH == 32 ? 96 : 512;
    __shared__ LogProbShared<TH, TOP ? kRoom : 1> shared[TH == 32 ? 8 : 1];
    auto& S = shared[TH == 32 ? threadIdx.x >> 5 : 0];
    const int tid = TH == 32 ? (int)threadIdx.x & 31 : (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long i = TH == 32 ? blockIdx.x * 8ll + (threadIdx.x >> 5) : (long long)blockIdx.x;
    if (i >= P.rows) return;  // (a whole warp; otherwise the grid has exactly the rows)
    const T* z = static_cast<const T*>(P.z) + i * P.ld;
    const RowPieces<T> row(z, P.C);
    const uint4* src = reinterpret_cast<const uint4*>(z + row.head);
    const int pieces = row.pieces;
    const int label = P.y ? P.y[i] : -1;
    float at_label = 0.f;
    if (label >= 0 && label < P.C) at_label = to_f32(z[label]);

    // ---- one pass: the sums of each thread, and its maximum
    Score a{-INFINITY, 0.f, 0.f};
    uint4 w[kAhead], next[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        if (tid + k * TH < pieces) next[k] = src[tid + k * TH];
    if (tid < row.edges) score_one(a, to_f32(z[row.edge(tid)]));
    for (int k0 = tid; k0 < pieces; k0 += kAhead * TH) {
        float m = a.m;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            w[k] = next[k];
            if (k0 + (kAhead + k) * TH < pieces) next[k] = src[k0 + (kAhead + k) * TH];
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (k0 + k * TH < pieces) m = score_max(m, score_piece_max<T>(w[k]));
        if (!(m <= a.m)) score_raise(a, m);
        const float base = score_base(a.m);
        Pair s(a.s, 0.f), t(a.t, 0.f);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (k0 + k * TH < pieces) score_piece<T>(w[k], Pair(-base), s, t);
        const float2 s2 = s.both(), t2 = t.both();
        a.s = s2.x + s2.y;
        a.t = t2.x + t2.y;
    }
    const float own = a.m;  // this thread's maximum
    if constexpr (TOP && TH > 32) S.lanes[warp][lane] = own;
    a = score_lanes(a);
    if constexpr (TH > 32) {
        if (lane == 0) S.part[warp] = a;
    }
    if constexpr (TOP) {
        if (tid == 0) S.owner_count = S.found_count = 0;
    }
    row_sync<TH>();
    if constexpr (TH > 32) {
        a = S.part[0];
#pragma unroll
        for (int k = 1; k < kWarps; ++k) a = score_join(a, S.part[k]);
    }
    const bool nothing = a.m == -INFINITY, broken = !(a.m < INFINITY);  // (no distribution; NaN or +Inf)
    const float nan = __uint_as_float(0x7FC00000u);
    const float log_s = broken ? nan : nothing ? 0.f : logf(a.s);
    if (tid == 0) {
        const float entropy = broken ? nan : nothing ? 0.f : log_s - a.t / a.s;
        if (P.logprob) P.logprob[i] = label < 0 || label >= P.C || nothing ? 0.f : (at_label - a.m) - log_s;
        if (P.entropy) P.entropy[i] = entropy;
        if (P.saved) {
            P.saved[3 * i] = a.m;
            P.saved[3 * i + 1] = log_s;
            P.saved[3 * i + 2] = entropy;
        }
    }
    if constexpr (!TOP) return;

    // ---- the alternatives
    const int top = P.top;
    uint32_t bound = 0;
    if (TH == 32 || warp == 0) {
        uint32_t g = rank_bits(own);
        if constexpr (TH > 32) {
            g = 0;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) g = max(g, rank_bits(S.lanes[k][lane]));
        }
        int rank = 0;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const uint32_t o = __shfl_sync(0xFFFFFFFFu, g, j);
            rank += o > g || (o == g && j < lane) ? 1 : 0;
        }
        bound = __shfl_sync(0xFFFFFFFFu, g, __ffs(__ballot_sync(0xFFFFFFFFu, rank == top - 1)) - 1);
        if (TH > 32 && lane == 0) S.bound = bound;
    }
    if constexpr (TH > 32) {
        __syncthreads();
        bound = S.bound;
    }
    if (rank_bits(own) >= bound) S.owners[atomicAdd(&S.owner_count, 1)] = tid;
    row_sync<TH>();
    // (a warp takes an owner at a time, each lane some of its pieces; lane 0 its edge, if it has one)
    auto consider = [&](float x, int c) {
        const uint32_t r = rank_bits(x);
        if (r >= bound) {
            const int n = atomicAdd(&S.found_count, 1);
            if (n < kRoom) S.found[n] = candidate(r, c);
        }
    };
    const int owners = S.owner_count;
    for (int k = warp; k < owners; k += kWarps) {
        const int u = S.owners[k];
        if (lane == 0 && u < row.edges) consider(to_f32(z[row.edge(u)]), row.edge(u));
        for (int p = u + lane * TH; p < pieces; p += 32 * TH) {
            const uint4 v = src[p];
            if (rank_bits(score_piece_max<T>(v)) < bound) continue;
            float x[VE];
            unpack_piece<T>(v, x);
#pragma unroll
            for (int e = 0; e < VE; ++e) consider(x[e], row.column(p) + e);
        }
    }
    row_sync<TH>();
    int found = S.found_count;
    if (found > kRoom) {
        row_sync<TH>();
        take_by_value<T>(z, P.C, top, S);
        found = top;
    }
    for (int k = tid; k < found; k += TH) {
        const unsigned long long mine = S.found[k];
        int rank = 0;
        for (int j = 0; j < found; ++j) rank += S.found[j] > mine ? 1 : 0;
        if (rank >= top) continue;
        const float x = rank_value((uint32_t)(mine >> 32));
        P.index[i * top + rank] = (int)(0xFFFFFFFFu - (uint32_t)mine);
        P.value[i * top + rank] = broken ? nan : nothing ? -INFINITY : (x - a.m) - log_s;
    }
}

// ---- gradient: each logit read once, its gradient written once
template <typename T, int TH>
__global__ void __launch_bounds__(TH == 32 ? 256 : TH) logprob_back_kernel(const __grid_constant__ LogProbParams P) {
    constexpr int VE = Piece<T>::kValues, kAhead = 2;
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
    const float k0 = nothing ? 0.f : -(a + b * entropy), k1 = nothing ? 0.f : -b, base = nothing ? 0.f : m;
    auto one = [&](float x, int c) {
        const float lp = fmaxf((x - base) - (nothing ? 0.f : log_s), kFarBelow), v = exp_fast(lp) * (k0 + k1 * lp);
        return c == label ? v + a : v;
    };
    if (tid < row.edges) dz[row.edge(tid)] = from_f32<T>(one(to_f32(z[row.edge(tid)]), row.edge(tid)));
    const Pair minus_m(-base), minus_s(nothing ? 0.f : -log_s), log2e(kLog2e), p0(k0), p1(k1);
    for (int q0 = tid; q0 < row.pieces; q0 += kAhead * TH) {
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
            store_piece(dz + c, out);
        }
    }
}

}  // namespace bmgdk
