// Directions of matrices by a polynomial of their singular values: X <- a X + (b A + c A^2) X, A = X X^T, some steps from X = u / |u|.
//
// A tensor is held as m x n with m <= n (transposed where it has more rows than columns): X in two f16 parts, H + 2^-11 L = 2^14 x.  The second
// part is held 2^11 times larger, so that it has all of f16's bits wherever the first one has: 22 bits of an element down to 2^-28 (|X| is near
// one), and below that to 2^-50.  (Both parts in one scale end at 2^-25 of the largest element: rows 1e-6 of the
// others' size would be 3e-3 off, and all of the direction 2e-2 after twelve steps.)  A = D + O and the polynomial B = b A + c A^2 are held
// as their diagonals in f32 and the rest in two f16 parts likewise (2^13 times the value, and as far as B allows), because the diagonals are the
// large part and what is rounded there changes whole rows:
//     A^2 outside the diagonal = (d_i + d_j) O_ij + (O O)_ij,     row i of the new X = (a + B_ii) X_i + (rest of B) X.
// The products take f16 on the matrix cores (train_gemm.h's tiles): first H L + L H, whose sum is then taken times 2^-11, on top of it H H; L L is left
// out, 2^-22 of the result at most.  One part alone in any of the products is not enough, not even for bf16 results: what it
// rounds off adds up over the steps to 4e-3 of the direction for matrices of low rank and to 4e-2 for exact rank one.
// Symmetric products form the tiles that reach the diagonal from below and store their results twice.
// Bound by the matrix cores for large matrices and by launches (three a step) for small ones.  One 4096 x 4096: a step's products 268
// (X X^T), 287 (square), 333 us (1.24 PFLOP/s in X's product, a large library product's rate; the symmetric ones leave half of the
// compute units idle); twelve of 1024 x 4096 215, 76, 324 us (0.95 PFLOP/s); two of 256 x 3136 11, 13, 13 us and 6 of a join.  Passes over the
// elements: 4096 x 4096, bf16, 15, 24, 18 us
#pragma once
#include "train_gemm.h"

#define TS_X 16384.0f       // of X: its singular values are below 2
#define TS_O 8192.0f        // of O, whose elements are below 4

struct SeriesProblem {
    const char *a[3], *b[3];
    size_t lda, ldb;       // bytes
    int M, N, K, nsrc, tiles_m, tiles_n;
    float *part;           // k axis in parts: [splits][M][ld_part]
    size_t ld_part;
    // epilogues
    _Float16 *o;           // GRAM: O; SQUARE: B's rest; APPLY: the new X
    const _Float16 *in;    // SQUARE: O; APPLY: X
    size_t apart;          // elements from the first part of o and of in to the second
    size_t ldo;            // elements, of o and in
    const float *diag;     // SQUARE: d; APPLY: a + B_ii
    float *diag_out;       // GRAM: d; SQUARE: a + B_ii
    float *last;           // APPLY: null, or the direction in f32 instead of o
    float ca, cb, cc;      // a, b, c
    float of_b;            // scale of B's rest: the largest power of two that keeps it inside f16
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
    l = (_Float16)((x - (float)h) * TS_LOW);
}
__device__ __forceinline__ void load_two(const _Float16 *p, size_t apart, float (&x)[8]) {
    float l[8];
    load_oct(p, x);
    load_oct(p + apart, l);
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] += l[e] * (1.0f / TS_LOW);
}
__device__ __forceinline__ void store_two(_Float16 *p, size_t apart, const float (&x)[8]) {
    float l[8];
#pragma unroll
    for (int e = 0; e < 8; e++) l[e] = (x[e] - (float)(_Float16)x[e]) * TS_LOW;
    store_oct(p, x);
    store_oct(p + apart, l);
}

// 8 columns of row m from n <= m on of a symmetric matrix without its diagonal: stored there and as a column
__device__ __forceinline__ void store_symmetric(const SeriesProblem &P, size_t m, int n, const float (&x)[8]) {
    _Float16 *row = P.o + m * P.ldo + n;
    if (n + 8 <= (int)m) store_two(row, P.apart, x);
#pragma unroll
    for (int e = 0; e < 8; e++) {
        if (n + e > (int)m) continue;
        _Float16 h, l;
        split16(n + e < (int)m ? x[e] : 0.0f, h, l);
        _Float16 *column = P.o + (size_t)(n + e) * P.ldo + m;
        *column = h;
        column[P.apart] = l;
        if (n + 8 > (int)m) {
            row[e] = h;
            row[P.apart + e] = l;
        }
    }
}

template <> struct SeriesEpilogue<EPI_GRAM> {
    static __device__ __forceinline__ void eight(const SeriesProblem &P, size_t m, int n, float (&v)[8]) {
#pragma unroll
        for (int e = 0; e < 8; e++) {
            v[e] *= TS_O / (TS_X * TS_X);
            if (n + e == (int)m) P.diag_out[m] = v[e] * (1.0f / TS_O);
        }
        store_symmetric(P, m, n, v);
    }
};
template <> struct SeriesEpilogue<EPI_SQUARE> {
    static __device__ __forceinline__ void eight(const SeriesProblem &P, size_t m, int n, float (&v)[8]) {
        float o[8];
        load_two(P.in + m * P.ldo + n, P.apart, o);
        const float d = P.diag[m];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            if (n + e > (int)m) continue;
            const float square = v[e] * (1.0f / TS_O);
            if (n + e == (int)m) P.diag_out[m] = P.ca + P.cb * d + P.cc * (d * d + square * (1.0f / TS_O));
            v[e] = (P.cb * o[e] + P.cc * ((d + P.diag[n + e]) * o[e] + square)) * (P.of_b / TS_O);
        }
        store_symmetric(P, m, n, v);
    }
};
template <> struct SeriesEpilogue<EPI_APPLY> {
    static __device__ __forceinline__ void eight(const SeriesProblem &P, size_t m, int n, float (&v)[8]) {
        float x[8];
        const size_t at = m * P.ldo + n;
        load_two(P.in + at, P.apart, x);
        const float d = P.diag[m], by = 1.0f / P.of_b;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            x[e] = d * x[e] + v[e] * by;
            if (P.last) x[e] *= 1.0f / TS_X;
            if (n + e >= P.N) x[e] = 0.0f;  // what pads a row stays zeros
        }
        if (P.last) store_oct(P.last + at, x);
        else store_two(P.o + at, P.apart, x);
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
    const float *part = P.part + m * P.ld_part + n;
    const size_t next = P.M * P.ld_part;
    float v[8] = {};
    // (four parts under way together: with one after the other 15 parts of 256 x 256 took 8.7 us)
    for (int s = 0; s < G.splits; s += 4) {
        float x[4][8];
#pragma unroll
        for (int k = 0; k < 4; k++) load_oct(part + min(s + k, G.splits - 1) * next, x[k]);
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (s + k < G.splits) v[e] = s + k ? v[e] + x[k][e] : x[k][e];
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
    _Float16 *o, *b;       // two parts of [side][ld_o]: their padding is set to zeros
    const float *direction;  // [side][ld]
    int64_t numel, per;    // per: elements of a workgroup of the first pass
    int rows, cols, ld, ld_o;
    float scale;           // lr times the tensor's
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

// u in units of its size: inverse as a power of two and the rest, so that neither leaves the range of f32 where inverse does
struct Unit {
    int exponent;
    float rest;
    __device__ __forceinline__ explicit Unit(double inverse) {
        exponent = 0;
        rest = (float)frexp(inverse, &exponent);
        if (!(inverse <= 1.7e308)) rest = (float)inverse;
    }
    __device__ __forceinline__ float of(float u) const { return ldexpf(u, exponent) * rest; }
};
__device__ __forceinline__ double series_inverse(const PassArgs &A, double squares) {
    const double size = sqrt(squares) + A.eps;
    return size < 1e-300 ? 0.0 : (double)TS_X / size;  // (f32 numbers that are not all zeros are larger)
}
// 64-bit sum over the workgroup
template <int THREADS> __device__ __forceinline__ double block_sum(double x, double (&sums)[THREADS]) {
    sums[threadIdx.x] = x;
    __syncthreads();
    for (int by = THREADS / 2; by; by /= 2) {
        if ((int)threadIdx.x < by) sums[threadIdx.x] += sums[threadIdx.x + by];
        __syncthreads();
    }
    return sums[0];
}

// Momentum, and the sum of squares of what is to be orthogonalised: in 64 bits (a gradient of 1e-25 has squares that f32 does not hold).
// A workgroup takes `per` neighbouring elements, 4096 at a time
template <class G> __global__ void __launch_bounds__(256) series_momentum_kernel(PassArgs A) {
    if (A.skip && *A.skip) return;
    const int i = pass_tensor(A);
    const PassTensor &t = A.t[i];
    const int64_t block = blockIdx.x - A.first[i], begin = block * t.per, end = begin + t.per < t.numel ? begin + t.per : t.numel;
    const G *g = (const G *)t.g;
    const bool g4 = at4(g), m4 = at4(t.m);
    double sum = 0.0;
    for (int64_t at = begin + 4 * threadIdx.x; at < end; at += 4096) {
        G gs[4][4];
        float ms[4][4];
#pragma unroll
        for (int k = 0; k < 4; k++) load4<false>(g, at + 1024 * k, end, g4, gs[k]);
        if (t.m)
#pragma unroll
            for (int k = 0; k < 4; k++) load4<false>(t.m, at + 1024 * k, end, m4, ms[k]);
#pragma unroll
        for (int k = 0; k < 4; k++) {
#pragma unroll
            for (int e = 0; e < 4; e++) {
                float u = (float)gs[k][e];
                if (t.m) {
                    ms[k][e] = momentum_of(A, ms[k][e], gs[k][e]);
                    u = direction_of(A, ms[k][e], gs[k][e]);
                }
                sum += (double)u * u;
            }
            if (t.m) store4<false>(t.m, at + 1024 * k, end, m4, ms[k]);
        }
    }
    __shared__ double sums[256];
    sum = block_sum<256>(sum, sums);
    if (threadIdx.x == 0) t.sums[block] = sum;
}

// 4 elements of a row from column c on, of which `left` exist (the others are zeros)
template <class T> __device__ __forceinline__ void get4(const T *p, int left, float (&x)[4]) {
    T v[4];
    if (left >= 4) __builtin_memcpy(v, p, sizeof(v));
    else
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = e < left ? p[e] : (T)0.0f;
#pragma unroll
    for (int e = 0; e < 4; e++) x[e] = (float)v[e];
}
template <class T> __device__ __forceinline__ void put4(T *p, int left, const float (&x)[4]) {
    T v[4];
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] = (T)x[e];
    if (left >= 4) __builtin_memcpy(p, v, sizeof(v));
    else
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (e < left) p[e] = v[e];
}

// A workgroup's 64 x 64 elements of a tensor, along its memory: rows r0 .. of memory, columns c0 ..
struct Square {
    int r0, c0;          // of memory
    bool tall;           // held transposed
    int side, length;    // as held
    __device__ __forceinline__ Square(const PassTensor &t, int block) {
        tall = t.rows > t.cols;
        side = tall ? t.cols : t.rows;
        length = tall ? t.rows : t.cols;
        const int across = (t.ld + 63) / 64, s0 = block / across * 64, l0 = block % across * 64;
        r0 = tall ? l0 : s0;
        c0 = tall ? s0 : l0;
    }
};

// X in its two parts from the momentum
template <class G> __global__ void __launch_bounds__(256) series_begin_kernel(PassArgs A) {
    const int i = pass_tensor(A);
    const PassTensor &t = A.t[i];
    const Square q(t, (int)(blockIdx.x - A.first[i]));
    __shared__ double sums[256];
    __shared__ float tile[64][65];
    // four rows of a column of 4 a thread; requested before the sums are added up
    const int r = threadIdx.x / 16, c = threadIdx.x % 16 * 4;
    float g[4][4], m[4][4];
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const int row = q.r0 + r + 16 * k;
        const size_t at = (size_t)row * t.cols + q.c0 + c;
        get4((const G *)t.g + at, row < t.rows ? t.cols - q.c0 - c : 0, g[k]);
        if (t.m) get4(t.m + at, row < t.rows ? t.cols - q.c0 - c : 0, m[k]);
    }
    double sum = 0.0;
    for (int b = threadIdx.x; b < t.blocks; b += 256) sum += t.sums[b];
    const Unit unit(series_inverse(A, block_sum<256>(sum, sums)));
#pragma unroll
    for (int k = 0; k < 4; k++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const float u = unit.of(t.m ? direction_of(A, m[k][e], g[k][e]) : g[k][e]);
            // (what lies beyond the matrix is 0 whatever the unit)
            const bool in = q.r0 + r + 16 * k < t.rows && q.c0 + c + e < t.cols;
            tile[q.tall ? c + e : r + 16 * k][q.tall ? r + 16 * k : c + e] = in ? u : 0.0f;
        }
    __syncthreads();
    const int s0 = q.tall ? q.c0 : q.r0, l0 = q.tall ? q.r0 : q.c0;
    const size_t apart = (size_t)q.side * t.ld;
#pragma unroll
    for (int k = 0; k < 2; k++) {
        const int row = threadIdx.x / 8 + 32 * k, at = threadIdx.x % 8 * 8;
        if (s0 + row >= q.side || l0 + at >= t.ld) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = tile[row][at + e];
        store_two(t.x + (size_t)(s0 + row) * t.ld + l0 + at, apart, v);
    }
    // the tensor's first tiles of a row clear what pads the symmetric matrices' rows
    if (l0 == 0 && t.ld_o > q.side)
        for (int k = threadIdx.x; k < 64 * 2; k += 256) {
            const int row = s0 + k % 64;
            if (row >= q.side) continue;
            for (int col = q.side; col < t.ld_o; col++) {
                const size_t at = ((size_t)(k / 64) * q.side + row) * t.ld_o + col;
                t.o[at] = t.b[at] = (_Float16)0.0f;
            }
        }
}

// 4 parameters along their directions, or the directions themselves (MOVE false)
template <class P, bool MOVE> __device__ __forceinline__ void series_move(const PassArgs &A, const PassTensor &t, size_t at, int left, const float (&d)[4]) {
    float p[4];
    if (MOVE) {
        get4((const P *)t.p + at, left, p);
#pragma unroll
        for (int e = 0; e < 4; e++) p[e] = p[e] * A.decay - d[e] * t.scale;
    }
    put4((P *)t.p + at, left, MOVE ? p : d);
    if (MOVE && t.copy) {
        if (A.copy_f16) put4((_Float16 *)t.copy + at, left, p);
        else put4((__bf16 *)t.copy + at, left, p);
    }
}
template <class P, bool MOVE> __global__ void __launch_bounds__(256) series_end_kernel(PassArgs A) {
    if (A.skip && *A.skip) return;
    const int i = pass_tensor(A);
    const PassTensor &t = A.t[i];
    const Square q(t, (int)(blockIdx.x - A.first[i]));
    __shared__ float tile[64][65];
    const int r = threadIdx.x / 16, c = threadIdx.x % 16 * 4, s0 = q.tall ? q.c0 : q.r0, l0 = q.tall ? q.r0 : q.c0;
    float d[4][4];
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const int row = s0 + r + 16 * k;
        get4(t.direction + (size_t)row * t.ld + l0 + c, row < q.side ? q.length - l0 - c : 0, d[k]);
    }
    if (q.tall) {
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
            for (int e = 0; e < 4; e++) tile[c + e][r + 16 * k] = d[k][e];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
            for (int e = 0; e < 4; e++) d[k][e] = tile[r + 16 * k][c + e];
    }
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const int row = q.r0 + r + 16 * k;
        if (row < t.rows && q.c0 + c < t.cols) series_move<P, MOVE>(A, t, (size_t)row * t.cols + q.c0 + c, t.cols - q.c0 - c, d[k]);
    }
}

// ---- matrices that fit the LDS of a compute unit: everything in one workgroup and one launch
// The same steps on 16 x 16 results a wave.  Rows and k indices (to a multiple of 32) that there are not are zeros in LDS and stay zeros; a row's
// elements begin 16 bytes further round the banks than the row's before.  The new X takes the old one's place: a wave takes 16 columns,
// and reads all of them before it writes.
// Bound by latency: three barriers a step, with a few LDS reads and products between them.  64 x 100, five steps: 32 us (in tiles, eighteen
// launches: 132)
#define TS_SMALL_LDS 151552
#define TS_SMALL_THREADS 1024
struct SmallSeries { int steps; float ca, cb, cc, of_b; };
__host__ __device__ __forceinline__ int small_ld(int n) { return (n + 31) / 32 * 32 + 8; }
inline size_t small_lds(int side, int length) {
    const size_t M = (side + 15) / 16 * 16, rows = (side + 31) / 32 * 32;
    return 4 * (rows * small_ld(length) + 2 * M * small_ld((int)M));
}
template <class P, class G, bool MOVE> __global__ void __launch_bounds__(TS_SMALL_THREADS) series_small_kernel(PassArgs A, SmallSeries S) {
    if (A.skip && *A.skip) return;
    const PassTensor &t = A.t[blockIdx.x];
    __shared__ __attribute__((aligned(1024))) char lds[TS_SMALL_LDS];
    __shared__ double sums[TS_SMALL_THREADS];
    __shared__ float d[64], e[64];
    TG_LDS(lds);
    const bool tall = t.rows > t.cols;
    const int side = tall ? t.cols : t.rows, length = tall ? t.rows : t.cols, tiles = (side + 15) / 16, M = 16 * tiles, ld = small_ld(length), ld_o = small_ld(M);
    const int x_apart = (M + 31) / 32 * 32 * ld, o_apart = M * ld_o;
    _Float16 *const X = (_Float16 *)lds, *const O = X + 2 * x_apart, *const B = O + 2 * o_apart;  // parts one behind the other
    const int lane = threadIdx.x & 63, wave = TG_UNIFORM((int)(threadIdx.x >> 6)), i = lane & 15, q = lane >> 4;
    constexpr int WAVES = TS_SMALL_THREADS / 64;
    for (int k = threadIdx.x; k < 2 * (x_apart + 2 * o_apart) / 8; k += TS_SMALL_THREADS) ((u32x4 *)lds)[k] = u32x4{0, 0, 0, 0};
    __syncthreads();
    // u, held as its word's halves where X's parts will be; momentum and size.  Eight elements of a thread are requested together
    const G *g = (const G *)t.g;
    const int numel = (int)t.numel;
    auto place = [&](int k) {
        const int r = k / t.cols, c = k - r * t.cols;
        return tall ? c * ld + r : r * ld + c;
    };
    double sum = 0.0;
    for (int first = threadIdx.x; first < numel; first += 8 * TS_SMALL_THREADS) {
        float u[8], m[8];
#pragma unroll
        for (int j = 0; j < 8; j++) u[j] = (float)g[min(first + j * TS_SMALL_THREADS, numel - 1)];
        if (t.m) {
#pragma unroll
            for (int j = 0; j < 8; j++) m[j] = t.m[min(first + j * TS_SMALL_THREADS, numel - 1)];
        }
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int k = first + j * TS_SMALL_THREADS;
            if (k >= numel) continue;
            if (t.m) {
                t.m[k] = m[j] = momentum_of(A, m[j], u[j]);
                u[j] = direction_of(A, m[j], u[j]);
            }
            sum += (double)u[j] * u[j];
            const unsigned word = __float_as_uint(u[j]);
            const int at = place(k);
            ((uint16_t *)X)[at] = (uint16_t)(word >> 16);
            ((uint16_t *)X)[x_apart + at] = (uint16_t)word;
        }
    }
    const Unit unit(series_inverse(A, block_sum<TS_SMALL_THREADS>(sum, sums)));
    for (int k = threadIdx.x; k < numel; k += TS_SMALL_THREADS) {
        const int at = place(k);
        const float u = __uint_as_float((unsigned)((uint16_t *)X)[at] << 16 | ((uint16_t *)X)[x_apart + at]);
        split16(unit.of(u), X[at], X[x_apart + at]);
    }
    // 16 bytes of a lane: row l % 16, k chunk l / 16 of rows along k
    auto fragment = [&](const _Float16 *p, int row0, int stride, int k) { return lds_read16((LdsPointer)(p + (row0 + i) * stride + k + 8 * q)); };
    // ... of rows of X as columns: column l % 16, k indices 8 (l / 16) .. + 7
    auto column = [&](const _Float16 *p, int n0, int k) {
        s16x4 h[2];
#pragma unroll
        for (int j = 0; j < 2; j++) h[j] = lds_read_transposed((LdsPointer)(p + (k + 8 * q + 4 * j + (i >> 2)) * ld + n0 + 4 * (i & 3)));
        u32x4 f;
        __builtin_memcpy(&f, h, 16);
        return f;
    };
    // sums of H H and of H L + L H
    auto with_low = [](f32x4 acc, f32x4 low) {
#pragma unroll
        for (int k = 0; k < 4; k++) acc[k] += low[k] * (1.0f / TS_LOW);
        return acc;
    };
    // 16 x 16 results of a symmetric product of rows along k: lane l has row l % 16, columns 4 (l / 16) .. + 3
    auto symmetric_tile = [&](const _Float16 *p, int apart, int stride, int row, int col, int K) {
        f32x4 acc = {0, 0, 0, 0}, low = {0, 0, 0, 0};
        for (int k = 0; k < K; k += 32) {
            const u32x4 a = fragment(p, col, stride, k), b = fragment(p, row, stride, k);
            acc = mma<_Float16>(a, b, acc);
            low = mma<_Float16>(a, fragment(p + apart, row, stride, k), low);
            low = mma<_Float16>(fragment(p + apart, col, stride, k), b, low);
        }
        return with_low(acc, low);
    };
    // four neighbouring columns of a row of a symmetric matrix, and as a column; those that reach the diagonal one by one
    auto put = [&](_Float16 *p, int row, int col, const float (&x)[4]) {
        _Float16 h[4], l[4];
#pragma unroll
        for (int k = 0; k < 4; k++) {
            split16(x[k], h[k], l[k]);
            if (col + k >= row) continue;
            p[(col + k) * ld_o + row] = h[k];
            p[o_apart + (col + k) * ld_o + row] = l[k];
            if (col + 3 >= row) {
                p[row * ld_o + col + k] = h[k];
                p[o_apart + row * ld_o + col + k] = l[k];
            }
        }
        if (col + 3 < row) {
            __builtin_memcpy(__builtin_assume_aligned(p + row * ld_o + col, 8), h, 8);
            __builtin_memcpy(__builtin_assume_aligned(p + o_apart + row * ld_o + col, 8), l, 8);
        }
    };
    auto four = [&](const _Float16 *p, int apart, float (&x)[4]) {
        _Float16 h[4], l[4];
        __builtin_memcpy(h, __builtin_assume_aligned(p, 8), 8);
        __builtin_memcpy(l, __builtin_assume_aligned(p + apart, 8), 8);
#pragma unroll
        for (int k = 0; k < 4; k++) x[k] = (float)h[k] + (float)l[k] * (1.0f / TS_LOW);
    };
    const int pairs = tiles * (tiles + 1) / 2, columns = (length + 15) / 16;
    const float by = 1.0f / S.of_b;
    for (int s = 0; s < S.steps; s++) {
        __syncthreads();
        for (int p = wave; p < pairs; p += WAVES) {
            int row, col;
            triangle_tile<1>(p, row, col);
            const f32x4 v = symmetric_tile(X, x_apart, ld, 16 * row, 16 * col, (length + 31) / 32 * 32);
            const int m = 16 * row + i, n = 16 * col + 4 * q;
            float x[4];
#pragma unroll
            for (int k = 0; k < 4; k++) {
                x[k] = v[k] * (TS_O / (TS_X * TS_X));
                if (n + k == m) d[m] = x[k] * (1.0f / TS_O);
            }
            put(O, m, n, x);
        }
        __syncthreads();
        for (int p = wave; p < pairs; p += WAVES) {
            int row, col;
            triangle_tile<1>(p, row, col);
            const f32x4 v = symmetric_tile(O, o_apart, ld_o, 16 * row, 16 * col, (M + 31) / 32 * 32);
            const int m = 16 * row + i, n = 16 * col + 4 * q;
            const float dm = d[m];
            float o[4];
            four(O + m * ld_o + n, o_apart, o);
#pragma unroll
            for (int k = 0; k < 4; k++) {
                const float square = v[k] * (1.0f / TS_O);
                if (n + k == m) e[m] = S.ca + S.cb * dm + S.cc * (dm * dm + square * (1.0f / TS_O));
                o[k] = (S.cb * o[k] + S.cc * ((dm + d[n + k]) * o[k] + square)) * (S.of_b / TS_O);
            }
            put(B, m, n, o);
        }
        __syncthreads();
        for (int c = wave; c < columns; c += WAVES) {
            u32x4 x[2][2];  // k steps, parts
#pragma unroll
            for (int k = 0; k < 2; k++)
                if (32 * k < M) {
                    x[k][0] = column(X, 16 * c, 32 * k);
                    x[k][1] = column(X + x_apart, 16 * c, 32 * k);
                }
            f32x4 acc[4];
#pragma unroll
            for (int r = 0; r < 4; r++) {
                f32x4 low = {0, 0, 0, 0};
                acc[r] = low;
                if (r >= tiles) continue;
#pragma unroll
                for (int k = 0; k < 2; k++)
                    if (32 * k < M) {
                        const u32x4 b = fragment(B, 16 * r, ld_o, 32 * k);
                        acc[r] = mma<_Float16>(x[k][0], b, acc[r]);
                        low = mma<_Float16>(x[k][1], b, low);
                        low = mma<_Float16>(x[k][0], fragment(B + o_apart, 16 * r, ld_o, 32 * k), low);
                    }
                acc[r] = with_low(acc[r], low);
            }
#pragma unroll
            for (int r = 0; r < 4; r++) {
                if (r >= tiles) continue;
                const int m = 16 * r + i;
                _Float16 *const at = X + m * ld + 16 * c + 4 * q;
                const float em = e[m];
                float old[4];
                four(at, x_apart, old);
                _Float16 h[4], l[4];
#pragma unroll
                for (int k = 0; k < 4; k++) split16(em * old[k] + acc[r][k] * by, h[k], l[k]);
                __builtin_memcpy(__builtin_assume_aligned(at, 8), h, 8);
                __builtin_memcpy(__builtin_assume_aligned(at + x_apart, 8), l, 8);
            }
        }
    }
    __syncthreads();
    const float size = 1.0f / TS_X;
    for (int first = threadIdx.x; first < numel; first += 8 * TS_SMALL_THREADS) {
        float p[8];
        if (MOVE)
#pragma unroll
            for (int j = 0; j < 8; j++) p[j] = (float)((const P *)t.p)[min(first + j * TS_SMALL_THREADS, numel - 1)];
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int k = first + j * TS_SMALL_THREADS;
            if (k >= numel) continue;
            const int at = place(k);
            const float v = ((float)X[at] + (float)X[x_apart + at] * (1.0f / TS_LOW)) * size, moved = MOVE ? p[j] * A.decay - v * t.scale : v;
            ((P *)t.p)[k] = (P)moved;
            if (MOVE && t.copy) {
                if (A.copy_f16) ((_Float16 *)t.copy)[k] = (_Float16)moved;
                else ((__bf16 *)t.copy)[k] = (__bf16)moved;
            }
        }
    }
}
