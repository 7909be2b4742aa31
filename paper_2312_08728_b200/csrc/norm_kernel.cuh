// Root-mean-square norm of rows with the residual's addition (bmgd_rms_norm_forward, bmgd_rms_norm_backward), and rows in 8 bits
// (its output there, bmgd_quantize_rows, bmgd_quantize_weight).
//
//     t = x + r rounded to the rows' type,  s = 1 / sqrt(mean_c t_c^2 + eps),  y_c = t_c s w_c
//     backward, g = dy w:  dt_c = dtotal_c + s (g_c - t_c s^2 mean(g t)),   dw_c = sum over rows of dy_c t_c s
//     8 bits:  a = max_c |y_c|,  scale = a / 127,  code_c = y_c (1 / a) 127 rounded to the nearest whole number
//
// The norm is that of the rounded sum: it is what the next block reads as its residual, what is kept for the backward pass, and so
// the gradients are those of the values that were computed.  Sums are fp32, squares of fp32 rows 64 bits.  What bounds it: memory, each value read and
// written once; rows are held in registers between the sum and its use.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>
#include <type_traits>

#include "activation.cuh"
#include "launch.cuh"
#include "values.cuh"

namespace bmgdk {

// Rows whose largest magnitude is below 2^-120 are zeros in 8 bits: 127 times its reciprocal would leave the range of fp32.  Beyond 2^126 the reciprocal is subnormal and
// good to 2^-22: 3e-5 of a code.
constexpr float kCodesLeast = 7.52316384526264e-37f;  // 2^-120

struct NormParams {
    const void *x, *residual, *weight;  // residual, weight: null for none
    void *total, *y;                    // total: null without a residual
    signed char* codes;                 // instead of y
    float *scale, *rstd;                // rstd: null if it is not wanted
    const void *dy, *dtotal;
    void *dx, *dweight;
    float* part;                        // backward: [gridDim.x][width], sums of each block's rows
    long long ld_x, ld_residual, ld_total, ld_y, ld_codes, ld_dy, ld_dtotal, ld_dx;
    long long rows;
    int width;
    int weight_f32;
    float eps, per_width;               // per_width: 1 / width
    int far;                            // results are not to stay in L2
};

// Sums of squares.  fp32 rows: in 64 bits, since their results are held to fp32 themselves (codes next to a border follow every bit).
template <typename T> struct SquareSum { typedef float type; };
template <> struct SquareSum<float> { typedef double type; };
__device__ __forceinline__ void add_square(float& sum, float t) { sum = fmaf(t, t, sum); }
__device__ __forceinline__ void add_square(double& sum, float t) { sum = fma((double)t, (double)t, sum); }
template <typename V>
__device__ __forceinline__ float root_factor(V sum, const NormParams& P) {
    if constexpr (std::is_same<V, double>::value) return rsqrtf((float)(sum / (double)P.width) + P.eps);
    else return rsqrtf(fmaf(sum, P.per_width, P.eps));
}

template <typename T>
__device__ __forceinline__ void load_weights(const void* weight, int f32, int c, float (&w)[Piece<T>::kValues]) {
    constexpr int VE = Piece<T>::kValues;
    if (!weight) {
#pragma unroll
        for (int e = 0; e < VE; ++e) w[e] = 1.f;
    } else if (f32 || sizeof(T) == 4) {
        const float* p = static_cast<const float*>(weight) + c;
        if (((uintptr_t)p & 15u) == 0) {
#pragma unroll
            for (int e = 0; e < VE; e += 4) {
                const float4 v = __ldca(reinterpret_cast<const float4*>(p + e));
                w[e] = v.x; w[e + 1] = v.y; w[e + 2] = v.z; w[e + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < VE; ++e) w[e] = __ldca(p + e);
        }
    } else {
        const T* p = static_cast<const T*>(weight) + c;
        if (((uintptr_t)p & 15u) == 0) {
            unpack_piece<T>(__ldca(reinterpret_cast<const uint4*>(p)), w);
        } else {
#pragma unroll
            for (int e = 0; e < VE; ++e) w[e] = to_f32(p[e]);
        }
    }
}
template <typename T>
__device__ __forceinline__ float load_weight(const void* weight, int f32, int c) {
    if (!weight) return 1.f;
    return f32 ? static_cast<const float*>(weight)[c] : to_f32(static_cast<const T*>(weight)[c]);
}

// The factor that takes a row's values to whole numbers, and its scale.  A row with NaN or Inf (top is one of them) has scale
// NaN and codes 0; so has what is computed from it.
struct RowCodes {
    float factor, scale;
    __device__ __forceinline__ explicit RowCodes(float top) {
        const bool fine = top < INFINITY, some = top >= kCodesLeast;
        factor = fine && some ? __fmul_rn(__frcp_rn(top), 127.f) : 0.f;
        scale = !fine ? __uint_as_float(0x7FC00000u) : some ? __fdiv_rn(top, 127.f) : 0.f;
    }
    // The code stands in the low byte: next to 1.5 2^23 the step of fp32 is one, so the sum is the whole number, rounded to nearest
    // (conversions take the exponentials' unit: 4096 x 11008 values 43 us with them).  |y factor| <= 127 (1 + 2^-23): no code leaves the range.
    __device__ __forceinline__ uint32_t bits(float y) const { return __float_as_uint(__fadd_rn(__fmul_rn(y, factor), 12582912.f)); }
    __device__ __forceinline__ signed char code(float y) const { return factor == 0.f ? (signed char)0 : (signed char)bits(y); }
};
template <int VE, bool ALIGNED = false>
__device__ __forceinline__ void store_codes(signed char* p, const RowCodes& rc, const float (&y)[VE]) {
    uint32_t w[VE / 4];
#pragma unroll
    for (int e = 0; e < VE; e += 4) {
        w[e / 4] = __byte_perm(__byte_perm(rc.bits(y[e]), rc.bits(y[e + 1]), 0x0040), __byte_perm(rc.bits(y[e + 2]), rc.bits(y[e + 3]), 0x0040), 0x5410);
        if (rc.factor == 0.f) w[e / 4] = 0;  // (also for NaN and Inf)
    }
    if (ALIGNED || ((uintptr_t)p & (VE - 1)) == 0) {
        if constexpr (VE == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(p) = w[0];
    } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) p[e] = (signed char)(w[e / 4] >> (8 * (e & 3)));
    }
}

// A value joined over the threads of a row, in a fixed order: a warp, or a whole block of any number of warps, whose spare cells are zero.
template <bool WARP, int OP, typename V>
__device__ __forceinline__ V join_threads(V v, V (&cells)[32]) {
    auto op = [](V a, V b) { if constexpr (OP == kJoinSum) return a + b; else return nan_max(a, b); };
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    if constexpr (!WARP) {
        if ((threadIdx.x & 31) == 0) cells[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0;  // (maxima here are of magnitudes)
        for (int k = 0; k < (int)(blockDim.x >> 5); k += 4) {
            V c[4];
            if constexpr (sizeof(V) == 4) *reinterpret_cast<float4*>(c) = *reinterpret_cast<const float4*>(cells + k);
            else for (int e = 0; e < 4; ++e) c[e] = cells[k + e];
            v = op(op(v, c[0]), op(c[1], op(c[2], c[3])));
        }
    }
    return v;
}

// ---- forward, rows held in registers: every thread has the same columns in every row that it meets, so that its weights stay in registers
// (read anew for each row they took four times the shared-memory cycles of the row itself: 8192 x 4096 31.5 us), and blocks go through the
// rows with the grid's stride, the next row under way while this one is summed up and written.  WARP: a warp to a row, eight rows to a block; otherwise
// as many threads as NV pieces each need.  ANY: rows that do not all start on 16-byte boundaries.  A block's rows are a multiple of eight apart (norm.cu sees to it), so
// all of them start at the same place within 16 bytes, in each tensor: the values before the first boundary of x (`head`) and behind its last piece go one each to the first
// threads, and tensors whose rows start elsewhere than x's are read and written value by value.
template <typename T, bool ANY>
struct Place {  // of a block's (a warp's) rows
    int head, pieces, edges;
    __device__ __forceinline__ Place(const T* x, int width) : head(0), pieces(width / Piece<T>::kValues), edges(0) {
        if constexpr (ANY) {
            const RowPieces<T> row(x, width);
            head = row.head;
            pieces = row.pieces;
            edges = row.edges;
        }
    }
    __device__ __forceinline__ int column(int piece) const { return head + piece * Piece<T>::kValues; }
    __device__ __forceinline__ int edge(int i) const { return i < head ? i : i + pieces * Piece<T>::kValues; }
    // (counted in pieces, not values, where that is possible: 4096 x 11008 values behind the gate 64 us otherwise, 50 so; by now 45)
    __device__ __forceinline__ uint4 load(const T* row, int piece) const {
        if constexpr (ANY) return load_piece(row + column(piece));
        else return __ldcs(reinterpret_cast<const uint4*>(row) + piece);
    }
    __device__ __forceinline__ void store(T* row, int piece, const uint4& w, bool far) const {
        if constexpr (ANY) store_piece(row + column(piece), w, far);
        else store16(reinterpret_cast<uint4*>(row) + piece, w, far);
    }
};

template <typename T, int NV, bool WARP, bool RES, bool CODES, bool ANY>
__global__ void __launch_bounds__(WARP ? 256 : 512, NV >= 4 ? 1 : 2) norm_flow_kernel(const __grid_constant__ NormParams P) {
    wait_for_previous_kernel();
    let_next_kernel_start();
    constexpr int VE = Piece<T>::kValues;
    constexpr bool kAhead = NV <= 4;  // (registers do not suffice for two rows of eight pieces, nor for their weights)
    typedef typename SquareSum<T>::type Sum;
    __shared__ __align__(16) Sum sums[2][32];
    __shared__ __align__(16) float tops[2][32];
    const int tid = WARP ? (int)threadIdx.x & 31 : (int)threadIdx.x, threads = WARP ? 32 : (int)blockDim.x;
    const long long step = (long long)gridDim.x * (WARP ? 8 : 1);
    if constexpr (!WARP) {
        for (int k = threadIdx.x; k < 64; k += blockDim.x) {
            (&sums[0][0])[k] = 0;
            (&tops[0][0])[k] = 0.f;
        }
        __syncthreads();
    }
    long long i = WARP ? blockIdx.x * 8ll + (threadIdx.x >> 5) : (long long)blockIdx.x;
    if (i >= P.rows) return;  // (a whole warp; otherwise there is a row for each block)
    const Place<T, ANY> place(static_cast<const T*>(P.x) + i * P.ld_x, P.width);
    const bool odd = ANY && tid < place.edges;
    const int at = odd ? place.edge(tid) : 0;
    float w[kAhead ? NV : 1][VE], edge_weight = odd ? load_weight<T>(P.weight, P.weight_f32, at) : 0.f;
    if constexpr (kAhead) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (tid + k * threads < place.pieces) load_weights<T>(P.weight, P.weight_f32, place.column(tid + k * threads), w[k]);
    }
    uint4 nx[NV], nr[RES ? NV : 1];
    float next_edge = 0.f, next_residual = 0.f;
    auto fetch = [&](long long row) {
        const T* x = static_cast<const T*>(P.x) + row * P.ld_x;
        const T* r = static_cast<const T*>(P.residual) + row * P.ld_residual;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (tid + k * threads < place.pieces) {
                nx[k] = place.load(x, tid + k * threads);
                if constexpr (RES) nr[k] = place.load(r, tid + k * threads);
            }
        if (odd) {
            next_edge = to_f32(x[at]);
            if constexpr (RES) next_residual = to_f32(r[at]);
        }
    };
    fetch(i);
    for (int turn = 0; i < P.rows; i += step, turn ^= 1) {
        Sum sum = 0;
        uint4 v[NV];
        float edge = next_edge;
        T* total = static_cast<T*>(P.total) + i * P.ld_total;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (tid + k * threads >= place.pieces) continue;
            float t[VE];
            v[k] = nx[k];
            unpack_piece<T>(v[k], t);
            if constexpr (RES) {
                float u[VE];
                unpack_piece<T>(nr[k], u);
#pragma unroll
                for (int e = 0; e < VE; ++e) t[e] += u[e];
                v[k] = pack_piece<T>(t);
                place.store(total, tid + k * threads, v[k], P.far != 0);
                unpack_piece<T>(v[k], t);
            }
#pragma unroll
            for (int e = 0; e < VE; ++e) add_square(sum, t[e]);
        }
        if (odd) {
            if constexpr (RES) {
                const T v1 = from_f32<T>(edge + next_residual);
                total[at] = v1;
                edge = to_f32(v1);
            }
            add_square(sum, edge);
        }
        if (kAhead && i + step < P.rows) fetch(i + step);
        const float s = root_factor(join_threads<WARP, kJoinSum>(sum, sums[turn]), P);
        if (P.rstd && tid == 0) P.rstd[i] = s;
        edge = edge * s * edge_weight;
        auto normed = [&](int k, float (&t)[VE]) {
            if constexpr (!kAhead) load_weights<T>(P.weight, P.weight_f32, place.column(tid + k * threads), w[0]);
            unpack_piece<T>(v[k], t);
#pragma unroll
            for (int e = 0; e < VE; ++e) t[e] = t[e] * s * w[kAhead ? k : 0][e];
        };
        if constexpr (!CODES) {
            T* y = static_cast<T*>(P.y) + i * P.ld_y;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (tid + k * threads >= place.pieces) continue;
                float t[VE];
                normed(k, t);
                place.store(y, tid + k * threads, pack_piece<T>(t), P.far != 0);
            }
            if (odd) y[at] = from_f32<T>(edge);
        } else {
            float top = odd ? fabsf(edge) : 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (tid + k * threads >= place.pieces) continue;
                float t[VE];
                normed(k, t);
#pragma unroll
                for (int e = 0; e < VE; ++e) top = nan_max(top, fabsf(t[e]));
            }
            const RowCodes rc(join_threads<WARP, kJoinMax>(top, tops[turn]));
            signed char* q = P.codes + i * P.ld_codes;
            if (tid == 0) P.scale[i] = rc.scale;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (tid + k * threads >= place.pieces) continue;
                float t[VE];
                normed(k, t);
                store_codes<VE, !ANY>(q + place.column(tid + k * threads), rc, t);
            }
            if (odd) q[at] = rc.code(edge);
        }
        if (!kAhead && i + step < P.rows) fetch(i + step);
    }
}

// ---- forward, rows of any length: a block of 1024 to a row, which is read again for each of the steps (from L2, mostly)
template <typename T, bool CODES>
__global__ void __launch_bounds__(1024) norm_long_kernel(const __grid_constant__ NormParams P) {
    wait_for_previous_kernel();
    let_next_kernel_start();
    constexpr int VE = Piece<T>::kValues, TH = 1024;
    __shared__ typename SquareSum<T>::type sums[TH / 32];
    __shared__ float tops[TH / 32];
    const int tid = threadIdx.x;
    const long long i = blockIdx.x;
    const T* x = static_cast<const T*>(P.x) + i * P.ld_x;
    const T* r = P.residual ? static_cast<const T*>(P.residual) + i * P.ld_residual : nullptr;
    T* total = static_cast<T*>(P.total) + i * P.ld_total;
    const RowPieces<T> row(x, P.width);
    const T* src = r ? total : x;  // where the sum is read from later (each thread reads what it has written)
    const bool odd = tid < row.edges;
    const int at = row.edge(tid);
    typename SquareSum<T>::type sum = 0;
    float t[VE], u[VE], edge = odd ? to_f32(x[at]) : 0.f;
    if (odd && r) {
        const T v1 = from_f32<T>(edge + to_f32(r[at]));
        total[at] = v1;
        edge = to_f32(v1);
    }
    for (int k = tid; k < row.pieces; k += TH) {
        const int c = row.column(k);
        uint4 w = load_piece(x + c);
        unpack_piece<T>(w, t);
        if (r) {
            unpack_piece<T>(load_piece(r + c), u);
#pragma unroll
            for (int e = 0; e < VE; ++e) t[e] += u[e];
            w = pack_piece<T>(t);
            store_piece(total + c, w);
            unpack_piece<T>(w, t);
        }
#pragma unroll
        for (int e = 0; e < VE; ++e) add_square(sum, t[e]);
    }
    add_square(sum, edge);
    const float s = root_factor(join_row<TH, kJoinSum>(sum, sums), P);
    if (P.rstd && tid == 0) P.rstd[i] = s;
    if (odd) edge *= s * load_weight<T>(P.weight, P.weight_f32, at);
    auto normed = [&](int c) {
        unpack_piece<T>(load_piece(src + c), t);
        load_weights<T>(P.weight, P.weight_f32, c, u);
#pragma unroll
        for (int e = 0; e < VE; ++e) t[e] = t[e] * s * u[e];
    };
    if constexpr (!CODES) {
        T* y = static_cast<T*>(P.y) + i * P.ld_y;
        for (int k = tid; k < row.pieces; k += TH) {
            normed(row.column(k));
            store_piece(y + row.column(k), pack_piece<T>(t));
        }
        if (odd) y[at] = from_f32<T>(edge);
    } else {
        float top = odd ? fabsf(edge) : 0.f;
        for (int k = tid; k < row.pieces; k += TH) {
            normed(row.column(k));
#pragma unroll
            for (int e = 0; e < VE; ++e) top = nan_max(top, fabsf(t[e]));
        }
        const RowCodes rc(join_row<TH, kJoinMax>(top, tops));
        signed char* q = P.codes + i * P.ld_codes;
        if (tid == 0) P.scale[i] = rc.scale;
        for (int k = tid; k < row.pieces; k += TH) {
            normed(row.column(k));
            store_codes<VE>(q + row.column(k), rc, t);
        }
        if (odd) q[at] = rc.code(edge);
    }
}

// ---- backward: as the forward pass, each thread adding up its columns' share of dw in registers; norm_weight_kernel adds the blocks' sums
// in their order, so equal calls give equal bits.
template <typename T, int NV, bool WARP, bool ANY>
__global__ void __launch_bounds__(WARP ? 256 : 512, WARP ? 2 : 1) norm_back_kernel(const __grid_constant__ NormParams P) {
    constexpr int VE = Piece<T>::kValues;
    constexpr bool kAhead = NV <= 2;  // the next row is under way while this one is summed up (not where registers do not suffice)
    __shared__ __align__(16) float cells[2][32];
    __shared__ float joined[WARP ? 8 : 1][WARP ? 32 * NV * VE + 2 * VE : 1];
    let_next_kernel_start();
    const int tid = WARP ? (int)threadIdx.x & 31 : (int)threadIdx.x, threads = WARP ? 32 : (int)blockDim.x;
    const long long step = (long long)gridDim.x * (WARP ? 8 : 1);
    if constexpr (!WARP) {
        for (int k = threadIdx.x; k < 64; k += blockDim.x) (&cells[0][0])[k] = 0.f;
        __syncthreads();
    }
    long long i = WARP ? blockIdx.x * 8ll + (threadIdx.x >> 5) : (long long)blockIdx.x;
    // (a warp without a row holds zeros for all columns)
    const Place<T, ANY> place(static_cast<const T*>(P.x) + (i < P.rows ? i : 0) * P.ld_x, P.width);
    const bool odd = ANY && tid < place.edges;
    const int at = odd ? place.edge(tid) : 0;
    float w[kAhead ? NV : 1][VE], dw[NV][VE] = {}, edge_weight = odd ? load_weight<T>(P.weight, P.weight_f32, at) : 0.f, edge_dw = 0.f;
    if constexpr (kAhead) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (tid + k * threads < place.pieces) load_weights<T>(P.weight, P.weight_f32, place.column(tid + k * threads), w[k]);
    }
    auto weights = [&](int k) -> float (&)[VE] {
        if constexpr (kAhead) return w[k];
        load_weights<T>(P.weight, P.weight_f32, place.column(tid + k * threads), w[0]);
        return w[0];
    };
    uint4 na[NV], nb[NV], nd[NV];
    float s = 0.f, ea = 0.f, eb = 0.f, ed = 0.f;
    auto fetch = [&](long long row) {
        const T* t = static_cast<const T*>(P.x) + row * P.ld_x;
        const T* dy = static_cast<const T*>(P.dy) + row * P.ld_dy;
        const T* dt = static_cast<const T*>(P.dtotal) + row * P.ld_dtotal;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (tid + k * threads >= place.pieces) continue;
            na[k] = place.load(t, tid + k * threads);
            nb[k] = place.load(dy, tid + k * threads);
            if (P.dtotal) nd[k] = place.load(dt, tid + k * threads);
        }
        if (odd) {
            ea = to_f32(t[at]);
            eb = to_f32(dy[at]);
            if (P.dtotal) ed = to_f32(dt[at]);
        }
        s = __ldg(P.rstd + row);
    };
    if (kAhead && i < P.rows) fetch(i);
    for (int turn = 0; i < P.rows; i += step, turn ^= 1) {
        if (!kAhead) fetch(i);
        uint4 a[NV], b[NV], d[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) { a[k] = na[k]; b[k] = nb[k]; d[k] = nd[k]; }
        const float si = s, a1 = ea, b1 = eb, d1 = ed;
        if (kAhead && i + step < P.rows) fetch(i + step);
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (tid + k * threads >= place.pieces) continue;
            float u[VE], v[VE];
            unpack_piece<T>(a[k], u);
            unpack_piece<T>(b[k], v);
            float (&wk)[VE] = weights(k);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float p = v[e] * (u[e] * si);
                sum = fmaf(p, wk[e], sum);
                dw[k][e] += p;
            }
        }
        if (odd) {
            const float p = b1 * (a1 * si);
            sum = fmaf(p, edge_weight, sum);
            edge_dw += p;
        }
        const float mean = join_threads<WARP, kJoinSum>(sum, cells[turn]) * P.per_width;
        T* dx = static_cast<T*>(P.dx) + i * P.ld_dx;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (tid + k * threads >= place.pieces) continue;
            float u[VE], v[VE];
            unpack_piece<T>(a[k], u);
            unpack_piece<T>(b[k], v);
            float (&wk)[VE] = weights(k);
#pragma unroll
            for (int e = 0; e < VE; ++e) v[e] = si * (v[e] * wk[e] - u[e] * si * mean);
            if (P.dtotal) {
                unpack_piece<T>(d[k], u);
#pragma unroll
                for (int e = 0; e < VE; ++e) v[e] += u[e];
            }
            place.store(dx, tid + k * threads, pack_piece<T>(v), P.far != 0);
        }
        if (odd) {
            const float v = si * (b1 * edge_weight - a1 * si * mean);
            dx[at] = from_f32<T>(P.dtotal ? v + d1 : v);
        }
    }
    if (!P.part) return;
    float* part = P.part + (long long)blockIdx.x * P.width;
    float* to = WARP ? joined[threadIdx.x >> 5] : part;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (tid + k * threads >= place.pieces) continue;
#pragma unroll
        for (int e = 0; e < VE; ++e) to[place.column(tid + k * threads) + e] = dw[k][e];
    }
    if (odd) to[at] = edge_dw;
    if constexpr (WARP) {  // the eight warps' sums, in their order
        __syncthreads();
        for (int c = threadIdx.x; c < P.width; c += 256) {
            float v = joined[0][c];
#pragma unroll
            for (int g = 1; g < 8; ++g) v += joined[g][c];
            part[c] = v;
        }
    }
}

// VE neighbouring values of a long row as they are held and moved: a piece, or one
template <typename T, int VE>
struct Columns;  // VE neighbouring values as they are held and moved
template <typename T>
struct Columns<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T* p) { v = __ldcs(p); }
    __device__ __forceinline__ void load_again(const T* p) { v = *p; }  // (what will be read again)
    __device__ __forceinline__ void unpack(float (&x)[1]) const { x[0] = to_f32(v); }
    static __device__ __forceinline__ void store(T* p, const float (&x)[1], bool) { *p = from_f32<T>(x[0]); }
    static __device__ __forceinline__ void weights(const void* w, int f32, int c, float (&x)[1]) { x[0] = load_weight<T>(w, f32, c); }
};
template <typename T, int VE>
struct Columns {
    static_assert(VE == Piece<T>::kValues, "a piece, or one value");
    uint4 v;
    __device__ __forceinline__ void load(const T* p) { v = __ldcs(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void load_again(const T* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void unpack(float (&x)[VE]) const { unpack_piece<T>(v, x); }
    static __device__ __forceinline__ void store(T* p, const float (&x)[VE], bool far) { store16(reinterpret_cast<uint4*>(p), pack_piece<T>(x), far); }
    static __device__ __forceinline__ void weights(const void* w, int f32, int c, float (&x)[VE]) { load_weights<T>(w, f32, c, x); }
};

// longer rows: read twice (the second time from L2), the columns' sums kept in shared memory where they fit (SUMS), else in the block's part of the workspace; each is
// only touched by the thread that adds to it
template <typename T, int VE, bool SUMS>
__global__ void __launch_bounds__(1024) norm_back_long_kernel(const __grid_constant__ NormParams P) {
    constexpr int TH = 1024;
    using Col = Columns<T, VE>;
    extern __shared__ __align__(16) float norm_sums[];
    __shared__ float cells[2][TH / 32];
    let_next_kernel_start();
    const int tid = threadIdx.x, count = P.width / VE;  // (VE divides it)
    float* const part = P.part ? P.part + (long long)blockIdx.x * P.width : nullptr;
    float* const dw = SUMS ? norm_sums : part;
    int turn = 0;
    for (long long i = blockIdx.x; i < P.rows; i += gridDim.x, turn ^= 1) {
        const T* t = static_cast<const T*>(P.x) + i * P.ld_x;
        const T* dy = static_cast<const T*>(P.dy) + i * P.ld_dy;
        const T* dt = static_cast<const T*>(P.dtotal) + i * P.ld_dtotal;
        T* dx = static_cast<T*>(P.dx) + i * P.ld_dx;
        const float s = __ldg(P.rstd + i);
        const bool first = i == blockIdx.x;
        float sum = 0.f;
#pragma unroll 2
        for (int k = tid; k < count; k += TH) {
            const int c = k * VE;
            Col a, b;
            float u[VE], v[VE], w[VE];
            a.load_again(t + c);
            b.load_again(dy + c);
            a.unpack(u);
            b.unpack(v);
            Col::weights(P.weight, P.weight_f32, c, w);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float p = v[e] * (u[e] * s);
                sum = fmaf(p, w[e], sum);
                if (part) dw[c + e] = first ? p : dw[c + e] + p;
            }
        }
        const float mean = join_row<TH, kJoinSum>(sum, cells[turn]) * P.per_width;
#pragma unroll 2
        for (int k = tid; k < count; k += TH) {
            const int c = k * VE;
            Col a, b;
            float u[VE], v[VE], w[VE];
            a.load(t + c);
            b.load(dy + c);
            a.unpack(u);
            b.unpack(v);
            Col::weights(P.weight, P.weight_f32, c, w);
#pragma unroll
            for (int e = 0; e < VE; ++e) v[e] = s * (v[e] * w[e] - u[e] * s * mean);
            if (P.dtotal) {
                a.load(dt + c);
                a.unpack(u);
#pragma unroll
                for (int e = 0; e < VE; ++e) v[e] += u[e];
            }
            Col::store(dx + c, v, P.far != 0);
        }
    }
    if (SUMS && part)
        for (int k = tid; k < count; k += TH)
#pragma unroll
            for (int e = 0; e < VE; ++e) part[k * VE + e] = dw[k * VE + e];
}

// dw from the blocks' sums: 32 columns to a block, 32 threads to a column
template <typename T>
__global__ void __launch_bounds__(1024) norm_weight_kernel(const float* part, int blocks, int width, void* dweight, int f32) {
    __shared__ float cells[32][33];
    wait_for_previous_kernel();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float v = 0.f;
    if (c < width) {
#pragma unroll 4
        for (int b = warp; b < blocks; b += 32) v += __ldcg(part + (long long)b * width + c);
    }
    cells[warp][lane] = v;
    __syncthreads();
    if (warp != 0 || c >= width) return;
    v = cells[0][lane];
#pragma unroll
    for (int k = 1; k < 32; ++k) v += cells[k][lane];
    if (f32) static_cast<float*>(dweight)[c] = v;
    else static_cast<T*>(dweight)[c] = from_f32<T>(v);
}

// ---------------------------------------------------------------- rows in 8 bits
// h = x, or act(gate) x; codes and scale as above.  A row is held as fp32 values between its maximum and its codes.
struct CodesParams {
    const void *x, *gate;  // gate: null for none
    signed char* codes;
    float* scale;
    long long ld_x, ld_gate, ld_codes, rows;
    int width, act;
};
// act(gate) as it is wanted here.  SiLU and sigmoid of 16-bit rows: exponential and reciprocal from the special unit, within (8 + 2 |g|) 2^-24 of the value; of fp32 rows the exact
// functions, because their codes are read against values of the same type, and next to a border a code follows every bit.  GELU: within (16 + 2 g^2) 2^-24 below zero.
template <typename T, int ACT>
__device__ __forceinline__ float gate_value(float g) {
    if constexpr (ACT == kActRelu) return g <= 0.f ? 0.f : g;
    float s;
    if constexpr (ACT == kActGelu) return g * gelu_share(g, s);
    if constexpr (sizeof(T) == 4) {
        s = __fdiv_rn(1.f, 1.f + expf(-g));
    } else {
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(g * -kLog2e));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.f + s));
    }
    return ACT == kActSigmoid ? s : g * s;
}
// h *= act(u), the activation chosen outside the loops
template <typename T, int N>
__device__ __forceinline__ void gate_values(int act, float (&h)[N], const float (&u)[N]) {
    switch (act) {
    case kActRelu:
#pragma unroll
        for (int e = 0; e < N; ++e) h[e] *= gate_value<T, kActRelu>(u[e]);
        break;
    case kActGelu:
#pragma unroll
        for (int e = 0; e < N; ++e) h[e] *= gate_value<T, kActGelu>(u[e]);
        break;
    case kActSigmoid:
#pragma unroll
        for (int e = 0; e < N; ++e) h[e] *= gate_value<T, kActSigmoid>(u[e]);
        break;
    default:
#pragma unroll
        for (int e = 0; e < N; ++e) h[e] *= gate_value<T, kActSilu>(u[e]);
    }
}
template <typename T>
__device__ __forceinline__ void gated_piece(const CodesParams& P, const uint4& x, const uint4& g, float (&h)[Piece<T>::kValues]) {
    unpack_piece<T>(x, h);
    if (P.gate) {
        float u[Piece<T>::kValues];
        unpack_piece<T>(g, u);
        gate_values<T>(P.act, h, u);
    }
}
template <typename T>
__device__ __forceinline__ float gated_one(const CodesParams& P, T x, const T* g) {
    float h[1] = {to_f32(x)};
    if (P.gate) {
        const float u[1] = {to_f32(*g)};
        gate_values<T>(P.act, h, u);
    }
    return h[0];
}
// as norm_flow_kernel
template <typename T, int NV, bool WARP, bool GATE, bool ANY>
__global__ void __launch_bounds__(WARP ? 256 : 384, NV == 6 ? 1 : 2) codes_flow_kernel(const __grid_constant__ CodesParams P) {
    wait_for_previous_kernel();
    let_next_kernel_start();
    constexpr int VE = Piece<T>::kValues;
    __shared__ __align__(16) float cells[2][32];
    const int tid = WARP ? (int)threadIdx.x & 31 : (int)threadIdx.x, threads = WARP ? 32 : (int)blockDim.x;
    const long long step = (long long)gridDim.x * (WARP ? 8 : 1);
    if constexpr (!WARP) {
        for (int k = threadIdx.x; k < 64; k += blockDim.x) (&cells[0][0])[k] = 0.f;
        __syncthreads();
    }
    long long i = WARP ? blockIdx.x * 8ll + (threadIdx.x >> 5) : (long long)blockIdx.x;
    if (i >= P.rows) return;  // (a whole warp; otherwise there is a row for each block)
    const Place<T, ANY> place(static_cast<const T*>(P.x) + i * P.ld_x, P.width);
    const bool odd = ANY && tid < place.edges;
    const int at = odd ? place.edge(tid) : 0;
    uint4 nx[NV], ng[GATE ? NV : 1];
    float next_edge = 0.f;
    auto fetch = [&](long long row) {
        const T* x = static_cast<const T*>(P.x) + row * P.ld_x;
        const T* g = static_cast<const T*>(P.gate) + row * P.ld_gate;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (tid + k * threads < place.pieces) {
                nx[k] = place.load(x, tid + k * threads);
                if constexpr (GATE) ng[k] = place.load(g, tid + k * threads);
            }
        if (odd) next_edge = gated_one(P, x[at], g + at);
    };
    fetch(i);
    for (int turn = 0; i < P.rows; i += step, turn ^= 1) {
        const float edge = next_edge;
        float h[NV][VE], top = fabsf(edge);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (tid + k * threads >= place.pieces) continue;
            unpack_piece<T>(nx[k], h[k]);
            if constexpr (GATE) {
                float u[VE];
                unpack_piece<T>(ng[k], u);
                gate_values<T>(P.act, h[k], u);
            }
#pragma unroll
            for (int e = 0; e < VE; ++e) top = nan_max(top, fabsf(h[k][e]));
        }
        if (i + step < P.rows) fetch(i + step);
        const RowCodes rc(join_threads<WARP, kJoinMax>(top, cells[turn]));
        signed char* q = P.codes + i * P.ld_codes;
        if (tid == 0) P.scale[i] = rc.scale;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (tid + k * threads < place.pieces) store_codes<VE, !ANY>(q + place.column(tid + k * threads), rc, h[k]);
        if (odd) q[at] = rc.code(edge);
    }
}
// rows of any length, read twice
template <typename T>
__global__ void __launch_bounds__(1024) codes_long_kernel(const __grid_constant__ CodesParams P) {
    wait_for_previous_kernel();
    let_next_kernel_start();
    constexpr int VE = Piece<T>::kValues, TH = 1024;
    __shared__ float cells[TH / 32];
    const int tid = threadIdx.x;
    const long long i = blockIdx.x;
    const T* x = static_cast<const T*>(P.x) + i * P.ld_x;
    const T* g = static_cast<const T*>(P.gate) + i * P.ld_gate;
    const RowPieces<T> row(x, P.width);
    const bool odd = tid < row.edges;
    const int at = row.edge(tid);
    float edge = 0.f, h[VE];
    if (odd) edge = gated_one(P, x[at], g + at);
    float top = fabsf(edge);
    auto read = [&](int c) { gated_piece<T>(P, load_piece(x + c), P.gate ? load_piece(g + c) : make_uint4(0, 0, 0, 0), h); };
    for (int k = tid; k < row.pieces; k += TH) {
        read(row.column(k));
#pragma unroll
        for (int e = 0; e < VE; ++e) top = nan_max(top, fabsf(h[e]));
    }
    const RowCodes rc(join_row<TH, kJoinMax>(top, cells));
    signed char* q = P.codes + i * P.ld_codes;
    if (tid == 0) P.scale[i] = rc.scale;
    for (int k = tid; k < row.pieces; k += TH) {
        read(row.column(k));
        store_codes<VE>(q + row.column(k), rc, h);
    }
    if (odd) q[at] = rc.code(edge);
}

// Weights [inputs][outputs] as codes [outputs][inputs] with a scale for each output: 32 outputs to a block, read once for their
// maxima and once more for the codes, which go through shared memory to stand along the inputs.
template <typename T>
__global__ void __launch_bounds__(1024) codes_weight_kernel(const T* __restrict__ w, long long ld_w, int inputs, int outputs,
                                                            signed char* __restrict__ codes, long long ld_codes, float* __restrict__ scale) {
    __shared__ float cells[32][33];
    __shared__ signed char tile[32][132];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float top = 0.f;
    if (c < outputs) {
#pragma unroll 4
        for (int k = warp; k < inputs; k += 32) top = nan_max(top, fabsf(to_f32(w[(long long)k * ld_w + c])));
    }
    cells[warp][lane] = top;
    __syncthreads();
    top = cells[0][lane];
#pragma unroll
    for (int k = 1; k < 32; ++k) top = nan_max(top, cells[k][lane]);
    const RowCodes rc(top);
    if (warp == 0 && c < outputs) scale[c] = rc.scale;
    for (int k0 = 0; k0 < inputs; k0 += 128) {
#pragma unroll
        for (int k = warp; k < 128; k += 32)
            tile[lane][k] = c < outputs && k0 + k < inputs ? rc.code(to_f32(w[(long long)(k0 + k) * ld_w + c])) : (signed char)0;
        __syncthreads();
        const int out = blockIdx.x * 32 + warp;
        if (out < outputs) {
#pragma unroll
            for (int k = lane; k < 128; k += 32)
                if (k0 + k < inputs) codes[(long long)out * ld_codes + k0 + k] = tile[warp][k];
        }
        __syncthreads();
    }
}

}  // namespace bmgdk
