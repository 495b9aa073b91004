// Products of few rows with a weight matrix, y = x W^T, for answering requests: the weights are read once, at whatever
// alignment their rows have, and nothing is copied, staged or joined by another launch.
//
// A workgroup takes 16 weight rows (GATE: 16 of each matrix) and 16 * MT rows of x; its waves share the k axis in runs of 128
// bytes a row.  Both operands come from memory as the fragments that the matrix cores take, 16 bytes a lane (row l % 16, chunk
// l / 16); the waves' sums meet in LDS and are added in their order.
// Bound by the weights' bytes and, at these sizes, by the latency of one trip to memory: hence many waves, each with all its
// loads of two or four runs in flight.  (Four runs of both matrices take the registers of a wave in four: 28 us instead of 24 for
// 64 f32 rows of 3136 -> 256.)
// Measured: bf16, one row of 1024 -> 4096 -> 1024: gate 7.4 us (16.8 MB), down 6.9 us (8.4 MB in 64 workgroups), of which a launch
// of this kernel takes 4 us with next to nothing to read; 7 rows of 999 -> 2731 -> 501 (f16, 2-byte alignment) 11 and 10 us.
#pragma once
#include "train_gemm.h"

struct RowsArgs {
    const char *x, *w[2];
    size_t ldx, ldw;  // bytes
    int M, N, K;
    EpiArgs epi;
};

// 16 bytes of a row from element k on; elements from K on are zeros
template <class T> __device__ __forceinline__ u32x4 row_chunk(const char *row, int k, int K) {
    constexpr int EPC = 16 / sizeof(T);
    const T *p = (const T *)row + k;
    u32x4 v = {0, 0, 0, 0};
    if (k + EPC <= K) __builtin_memcpy(&v, p, 16);
    else if (k < K) {
        T e[EPC];
#pragma unroll
        for (int j = 0; j < EPC; j++) e[j] = k + j < K ? p[j] : (T)0.0f;
        __builtin_memcpy(&v, e, 16);
    }
    return v;
}

template <class T, int EPI, int MT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) rows_kernel(RowsArgs R) {
    constexpr int MATS = EPI == EPI_GATE ? 2 : 1, EPC = 16 / sizeof(T), RUN = 128 / sizeof(T);
    __shared__ f32x4 sums[WAVES][MATS][MT][64];
    const int lane = threadIdx.x & 63, wave = TG_UNIFORM((int)(threadIdx.x >> 6)), i = lane & 15, q = lane >> 4;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * MT;
    // rows beyond the end repeat the last one: their results are not stored
    const char *w[MATS], *x[MT];
#pragma unroll
    for (int a = 0; a < MATS; a++) w[a] = R.w[a] + (size_t)min(n0 + i, R.N - 1) * R.ldw;
#pragma unroll
    for (int t = 0; t < MT; t++) x[t] = R.x + (size_t)min(m0 + 16 * t + i, R.M - 1) * R.ldx;
    f32x4 acc[MATS][MT];
#pragma unroll
    for (int a = 0; a < MATS; a++)
#pragma unroll
        for (int t = 0; t < MT; t++) acc[a][t] = f32x4{0, 0, 0, 0};
    // a run of 128 bytes a row: two sub-steps of four chunks
    struct Run { u32x4 w[MATS][2], x[MT][2]; };
    auto load = [&](Run &f, int k0) {  // all of it exists
#pragma unroll
        for (int s = 0; s < 2; s++) {
            const int k = k0 + (4 * s + q) * EPC;
#pragma unroll
            for (int a = 0; a < MATS; a++) __builtin_memcpy(&f.w[a][s], w[a] + (size_t)k * sizeof(T), 16);
#pragma unroll
            for (int t = 0; t < MT; t++) __builtin_memcpy(&f.x[t][s], x[t] + (size_t)k * sizeof(T), 16);
        }
    };
    auto load_end = [&](Run &f, int k0) {  // some of it, or nothing: zeros
        if (k0 >= R.K) {
            f = Run{};
            return;
        }
#pragma unroll
        for (int s = 0; s < 2; s++) {
            const int k = k0 + (4 * s + q) * EPC;
#pragma unroll
            for (int a = 0; a < MATS; a++) f.w[a][s] = row_chunk<T>(w[a], k, R.K);
#pragma unroll
            for (int t = 0; t < MT; t++) f.x[t][s] = row_chunk<T>(x[t], k, R.K);
        }
    };
    auto multiply = [&](const Run &f) {
#pragma unroll
        for (int s = 0; s < 2; s++)
#pragma unroll
            for (int a = 0; a < MATS; a++)
#pragma unroll
                for (int t = 0; t < MT; t++) acc[a][t] = mma<T>(f.w[a][s], f.x[t][s], acc[a][t]);
    };
    constexpr int AHEAD = MATS + MT <= 2 ? 4 : 2;  // runs whose loads are under way together
    for (int k0 = wave * RUN; k0 < R.K; k0 += AHEAD * WAVES * RUN) {
        Run f[AHEAD];
#pragma unroll
        for (int r = 0; r < AHEAD; r++) {
            const int kr = k0 + r * WAVES * RUN;
            if (kr + RUN <= R.K) load(f[r], kr);
            else load_end(f[r], kr);
        }
#pragma unroll
        for (int r = 0; r < AHEAD; r++) multiply(f[r]);
    }
#pragma unroll
    for (int a = 0; a < MATS; a++)
#pragma unroll
        for (int t = 0; t < MT; t++) sums[wave][a][t][lane] = acc[a][t];
    __syncthreads();
    // lane l's sums are row l % 16's columns 4*(l/16) .. +3: a thread takes 8 columns of a row
    if (threadIdx.x >= 32 * MT) return;
    const int t = threadIdx.x / 32, row = threadIdx.x % 16, half = threadIdx.x / 16 % 2, m = m0 + 16 * t + row, n = n0 + 8 * half;
    if (m >= R.M || n >= R.N) return;
    float v[2][8];
#pragma unroll
    for (int a = 0; a < MATS; a++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
            f32x4 s = sums[0][a][t][(2 * half + e) * 16 + row];
#pragma unroll
            for (int k = 1; k < WAVES; k++) s += sums[k][a][t][(2 * half + e) * 16 + row];
#pragma unroll
            for (int j = 0; j < 4; j++) v[a][4 * e + j] = s[j];
        }
    epilogue8<T, EPI>(R.epi, m, n, v[0], v[MATS - 1]);
}
