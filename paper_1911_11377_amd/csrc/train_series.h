// Directions of matrices by a polynomial of their singular values: X <- a X + (b A + c A^2) X, A = X X^T, some steps from X = u / |u|.
//
// A tensor is held as m x n with m <= n (transposed where it has more rows than columns): X in two f16 parts, H + L = S x with S a power of
// two near sqrt(m n), so that elements of the usual size 1 / sqrt(m n) are near one: their two parts have 22 bits, and S times the
// largest singular value stays inside f16.  A = D + O and the polynomial B = b A + c A^2 are held as their diagonals in f32 and the
// rest in f16 (256 times the value), because the diagonals are the large part and what is rounded there changes whole rows:
//     A^2 outside the diagonal = (d_i + d_j) O_ij + (O O)_ij,     row i of the new X = (a + B_ii) X_i + (rest of B) X.
// The products take f16 on the matrix cores (train_gemm.h's tiles).  PARTS == 1: the upper parts alone, O and B's rest in one part; X itself keeps
// both through the sum, so rounding errors do not grow from step to step: 4e-4 - 9e-4 of the direction's size for gradients of any
// spectrum (X in one part: up to 4e-2 on matrices of low rank).  PARTS == 2: H H + H L + L H of two parts each, 22 bits: 1e-7 - 7e-6,
// less than sums in f32 add.  Symmetric products form the tiles that reach the diagonal from below and store their results twice.
// Bound by the matrix cores for large matrices and by launches (three a step) for small ones.
#pragma once
#include "train_gemm.h"

#define TS_SCALE 256.0f  // of O and of B's rest

struct SeriesProblem {
    const char *a[3], *b[3];
    size_t lda, ldb;       // bytes
    int M, N, K, nsrc, tiles_m, tiles_n;
    float *part;           // k axis in parts: [splits][M][ld_part]
    size_t ld_part;
    // epilogues
    _Float16 *o;           // GRAM: O; SQUARE: B's rest; APPLY: the new X
    const _Float16 *in;    // SQUARE: O; APPLY: X
    size_t o_apart, in_apart;  // elements from the first part to the second
    size_t ldo;            // elements, of o and in
    const float *diag;     // SQUARE: d; APPLY: a + B_ii
    float *diag_out;       // GRAM: d; SQUARE: a + B_ii
    float *last;           // APPLY: null, or the direction in f32 instead of o
    float scale;           // GRAM: TS_SCALE / S^2; APPLY, last: 1 / S
    int parts;             // of o (GRAM, SQUARE)
    float ca, cb, cc;      // a, b, c
};

#define TS_PROBLEMS 16
struct SeriesArgs {
    typedef SeriesProblem Problem;
    SeriesProblem p[TS_PROBLEMS];
    int first[TS_PROBLEMS + 1];
    int n_problems, splits;
};
static_assert(sizeof(SeriesArgs) <= 4096, "kernel arguments");

__device__ __forceinline__ void split16(float x, _Float16 &h, _Float16 &l) {
    h = (_Float16)x;
    l = (_Float16)(x - (float)h);
}
__device__ __forceinline__ void load_parts(const _Float16 *p, size_t apart, int parts, float (&x)[8]) {
    load_oct(p, x);
    if (parts > 1) {
        float l[8];
        load_oct(p + apart, l);
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] += l[e];
    }
}
__device__ __forceinline__ void store_two(_Float16 *p, size_t apart, const float (&x)[8]) {
    float l[8];
#pragma unroll
    for (int e = 0; e < 8; e++) l[e] = x[e] - (float)(_Float16)x[e];
    store_oct(p, x);
    store_oct(p + apart, l);
}

// 8 columns of row m from n <= m on of a symmetric matrix without its diagonal: stored there and as a column
__device__ __forceinline__ void store_symmetric(const SeriesProblem &P, size_t m, int n, const float (&x)[8]) {
    _Float16 *row = P.o + m * P.ldo + n;
    if (n + 8 <= (int)m) {
        if (P.parts > 1) store_two(row, P.o_apart, x);
        else store_oct(row, x);
    }
#pragma unroll
    for (int e = 0; e < 8; e++) {
        if (n + e > (int)m) continue;
        _Float16 h, l;
        split16(n + e < (int)m ? x[e] : 0.0f, h, l);
        _Float16 *column = P.o + (size_t)(n + e) * P.ldo + m;
        *column = h;
        if (P.parts > 1) column[P.o_apart] = l;
        if (n + 8 > (int)m) {
            row[e] = h;
            if (P.parts > 1) row[P.o_apart + e] = l;
        }
    }
}

template <> struct SeriesEpilogue<EPI_GRAM> {
    static __device__ __forceinline__ void eight(const SeriesProblem &P, size_t m, int n, float (&v)[8]) {
#pragma unroll
        for (int e = 0; e < 8; e++) {
            v[e] *= P.scale;
            if (n + e == (int)m) P.diag_out[m] = v[e] * (1.0f / TS_SCALE);
        }
        store_symmetric(P, m, n, v);
    }
};
template <> struct SeriesEpilogue<EPI_SQUARE> {
    static __device__ __forceinline__ void eight(const SeriesProblem &P, size_t m, int n, float (&v)[8]) {
        float o[8];
        load_parts(P.in + m * P.ldo + n, P.in_apart, P.parts, o);
        const float d = P.diag[m];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            if (n + e > (int)m) continue;
            const float square = v[e] * (1.0f / TS_SCALE);
            if (n + e == (int)m) P.diag_out[m] = P.ca + P.cb * d + P.cc * (d * d + square * (1.0f / TS_SCALE));
            v[e] = P.cb * o[e] + P.cc * ((d + P.diag[n + e]) * o[e] + square);
        }
        store_symmetric(P, m, n, v);
    }
};
template <> struct SeriesEpilogue<EPI_APPLY> {
    static __device__ __forceinline__ void eight(const SeriesProblem &P, size_t m, int n, float (&v)[8]) {
        float x[8];
        const size_t at = m * P.ldo + n;
        load_parts(P.in + at, P.in_apart, 2, x);
        const float d = P.diag[m];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            x[e] = d * x[e] + v[e] * (1.0f / TS_SCALE);
            if (P.last) x[e] *= P.scale;
            if (n + e >= P.N) x[e] = 0.0f;  // what pads a row stays zeros
        }
        if (P.last) store_oct(P.last + at, x);
        else store_two(P.o + at, P.o_apart, x);
    }
};

// Sum of the parts of a split k axis, always in the same order, and the epilogue
template <int EPI> __global__ void __launch_bounds__(256) series_join_kernel(SeriesArgs G) {
    const SeriesProblem &P = G.p[blockIdx.y];
    const size_t octs = P.ld_part / 8, id = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= octs * P.M) return;
    const size_t m = id / octs;
    const int n = (int)(id % octs) * 8;
    if (symmetric(EPI) && n > (int)m) return;
    float v[8];
    for (int s = 0; s < G.splits; s++) {
        float x[8];
        load_oct(P.part + ((size_t)s * P.M + m) * P.ld_part + n, x);
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = s ? v[e] + x[e] : x[e];
    }
    SeriesEpilogue<EPI>::eight(P, m, n, v);
}

// ---- passes over the tensors' elements
struct PassTensor {
    char *p;               // parameters, or where the direction goes
    const char *g;         // gradients, or the matrix itself
    float *m;              // momentum; null: the matrix itself
    char *copy;
    double *sums;          // of squares, one a workgroup of the first pass
    _Float16 *x;           // two parts of [side][ld]
    _Float16 *o, *b;       // [parts][side][ld_o]: their padding is set to zeros
    const float *direction;  // [side][ld]
    int64_t numel;
    int rows, cols, ld, ld_o, parts;
    float S, scale;        // scale: lr times the tensor's
    int blocks;            // workgroups of the first pass
};
#define TS_TENSORS 24
struct PassArgs {
    PassTensor t[TS_TENSORS];
    unsigned first[TS_TENSORS + 1];
    int n, g_dtype, copy_f16, nesterov;
    float momentum, rest, grad_scale, decay;
    double eps;
    const int *skip;
};
static_assert(sizeof(PassArgs) <= 4096, "kernel arguments");

__device__ __forceinline__ int pass_tensor(const PassArgs &A) {
    int lo = 0, hi = A.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (A.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}
template <class G> __device__ __forceinline__ float momentum_of(const PassArgs &A, float m, G g) { return m * A.momentum + (float)g * A.grad_scale * A.rest; }
// u from the momentum after its update
template <class G> __device__ __forceinline__ float direction_of(const PassArgs &A, float m, G g) { return A.nesterov ? m * A.momentum + (float)g * A.grad_scale * A.rest : m; }

// Momentum, and the sum of squares of what is to be orthogonalised: in 64 bits (a gradient of 1e-25 has squares that f32 does not hold)
#define TS_CHUNK 16384
template <class G> __global__ void __launch_bounds__(256) series_momentum_kernel(PassArgs A) {
    if (A.skip && *A.skip) return;
    const PassTensor &t = A.t[pass_tensor(A)];
    const unsigned block = blockIdx.x - A.first[pass_tensor(A)];
    const int64_t begin = (int64_t)block * TS_CHUNK, end = begin + TS_CHUNK < t.numel ? begin + TS_CHUNK : t.numel;
    const G *g = (const G *)t.g;
    double sum = 0.0;
    for (int64_t i = begin + threadIdx.x; i < end; i += 256) {
        float u = (float)g[i];
        if (t.m) {
            const float m = momentum_of(A, t.m[i], g[i]);
            t.m[i] = m;
            u = direction_of(A, m, g[i]);
        }
        sum += (double)u * u;
    }
    __shared__ double sums[256];
    sums[threadIdx.x] = sum;
    __syncthreads();
    for (int by = 128; by; by /= 2) {
        if ((int)threadIdx.x < by) sums[threadIdx.x] += sums[threadIdx.x + by];
        __syncthreads();
    }
    if (threadIdx.x == 0) t.sums[block] = sums[0];
}

// X in its two parts from the momentum; 64 x 64 elements a workgroup
template <class G> __global__ void __launch_bounds__(256) series_begin_kernel(PassArgs A) {
    const int i = pass_tensor(A);
    const PassTensor &t = A.t[i];
    __shared__ double sums[256];
    __shared__ float tile[64][65];
    double sum = 0.0;
    for (int b = threadIdx.x; b < t.blocks; b += 256) sum += t.sums[b];
    sums[threadIdx.x] = sum;
    __syncthreads();
    for (int by = 128; by; by /= 2) {
        if ((int)threadIdx.x < by) sums[threadIdx.x] += sums[threadIdx.x + by];
        __syncthreads();
    }
    const double size = sqrt(sums[0]) + A.eps, inverse = size == 0.0 ? 0.0 : (double)t.S / size;
    // tiles of the held orientation: side x length
    const bool tall = t.rows > t.cols;
    const int side = tall ? t.cols : t.rows, length = tall ? t.rows : t.cols, across = (t.ld + 63) / 64;
    const int block = (int)(blockIdx.x - A.first[i]), r0 = block / across * 64, c0 = block % across * 64;
    const G *g = (const G *)t.g;
    // what is read lies along memory: rows of the held tile, or (tall) its columns
    for (int k = threadIdx.x; k < 4096; k += 256) {
        const int along = k & 63, over = k >> 6, r = tall ? r0 + along : r0 + over, c = tall ? c0 + over : c0 + along;
        float u = 0.0f;
        if (r < side && c < length) {
            const size_t at = tall ? (size_t)c * t.cols + r : (size_t)r * t.cols + c;
            u = t.m ? direction_of(A, t.m[at], g[at]) : (float)g[at];
            u = (float)((double)u * inverse);
        }
        tile[tall ? along : over][tall ? over : along] = u;
    }
    __syncthreads();
    const size_t apart = (size_t)side * t.ld;
    for (int k = threadIdx.x; k < 512; k += 256) {
        const int r = k / 8, c = k % 8 * 8;
        if (r0 + r >= side || c0 + c >= t.ld) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = tile[r][c + e];
        store_two(t.x + (size_t)(r0 + r) * t.ld + c0 + c, apart, v);
    }
    // the tensor's first tiles of a row clear what pads the symmetric matrices' rows
    if (c0 == 0 && t.ld_o > side)
        for (int k = threadIdx.x; k < 64 * t.parts; k += 256) {
            const int r = r0 + k % 64;
            if (r >= side) continue;
            for (int c = side; c < t.ld_o; c++) {
                const size_t at = ((size_t)(k / 64) * side + r) * t.ld_o + c;
                t.o[at] = t.b[at] = (_Float16)0.0f;
            }
        }
}

// Parameters along the direction, or the direction itself (MOVE false); 64 x 64 elements a workgroup
template <class P, bool MOVE> __global__ void __launch_bounds__(256) series_end_kernel(PassArgs A) {
    if (A.skip && *A.skip) return;
    const int i = pass_tensor(A);
    const PassTensor &t = A.t[i];
    __shared__ float tile[64][65];
    const bool tall = t.rows > t.cols;
    const int side = tall ? t.cols : t.rows, length = tall ? t.rows : t.cols, across = (t.ld + 63) / 64;
    const int block = (int)(blockIdx.x - A.first[i]), r0 = block / across * 64, c0 = block % across * 64;
    if (tall) {
        for (int k = threadIdx.x; k < 4096; k += 256) {
            const int c = k & 63, r = k >> 6;
            tile[r][c] = r0 + r < side && c0 + c < length ? t.direction[(size_t)(r0 + r) * t.ld + c0 + c] : 0.0f;
        }
        __syncthreads();
    }
    for (int k = threadIdx.x; k < 4096; k += 256) {
        const int along = k & 63, over = k >> 6, r = tall ? along : over, c = tall ? over : along;
        if (r0 + r >= side || c0 + c >= length) continue;
        const float d = tall ? tile[r][c] : t.direction[(size_t)(r0 + r) * t.ld + c0 + c];
        const size_t at = tall ? (size_t)(c0 + c) * t.cols + r0 + r : (size_t)(r0 + r) * t.cols + c0 + c;
        P *p = (P *)t.p + at;
        const float q = MOVE ? (float)*p * A.decay - d * t.scale : d;
        *p = (P)q;
        if (MOVE && t.copy) {
            if (A.copy_f16) ((_Float16 *)t.copy)[at] = (_Float16)q;
            else ((__bf16 *)t.copy)[at] = (__bf16)q;
        }
    }
}
