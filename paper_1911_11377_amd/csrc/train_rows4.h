// Products of few rows with a matrix in 4 bits, y[m][o] = sum over groups G of scale[o][G] * (sum over k in G of code(o, k) x(m, k)): the codes
// are read once, 16 bytes a lane.
//
// A workgroup takes 16 rows of the matrix (GATE: 16 of each of two) and 16 * MT rows of x; its waves share the k axis in runs of 128.  Lane l
// reads 32 codes of row l % 16 from k0 + 32 (l / 16) on; four lanes of a row exchange words, so that each holds what a step of the matrix
// cores takes of it: 8 codes from k0 + 32 s + 8 (l / 16) on for step s.  Codes become bf16 or f16 exactly (in sixteenths: that is what the
// conversion gives), a group's sum stays in f32 and is scaled there: a scaled weight rounded to 16 bits would cost three decimal
// places of four.  x: 16-bit as it is, f32 in three bf16 parts, cut as it is read; h between the block's products in two or three bf16 parts.
// The waves' sums meet in LDS and are added in their order.
// Bound by the codes' bytes and, for small matrices, by the latency of one trip to memory.
#pragma once
#include "train_rows.h"

struct Rows4Args {
    const char *x;
    const uint8_t *codes[2];
    const char *scales[2];
    size_t ldx, ldc, lds;   // bytes; lds: elements of a row of scales
    size_t x_apart;         // bytes from one part of x to the next
    int M, N, K, group_shift;  // group = 32 << group_shift
    EpiArgs epi;
    char *h;                // GATE: act(g) u in bf16 parts, [parts][M][ldh]
    size_t ldh, h_apart;    // elements
    int h_parts;
};

#ifdef CKKSMI_EMULATE
#define code_to_float emu_code_to_float
#define exchange_words emu_exchange_words
#else
// the lowest 4 bits of c as a number from -8 to 7, in sixteenths
__device__ __forceinline__ float code_to_float(unsigned c) { return __builtin_amdgcn_cvt_off_f32_i4((int)c); }
// word s of the lane in row q of 16 lanes <-> word q of the lane in row s
__device__ __forceinline__ u32x4 exchange_words(u32x4 w) {
    // halves of the wave, words two apart; then rows of 16 within a half, neighbouring words
    auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
    auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return u32x4{c[0], c[1], d[0], d[1]};
}
#endif

// 8 codes as T, in sixteenths
template <class T> __device__ __forceinline__ u32x4 codes8(unsigned w) {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; e++) f[e] = code_to_float(w >> (4 * e));
    u32x4 o;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        if constexpr (__is_same(T, __bf16)) o[e] = __float_as_uint(f[2 * e]) >> 16 | (__float_as_uint(f[2 * e + 1]) & 0xffff0000u);
        else {
            struct { _Float16 low, high; } p = {(_Float16)f[2 * e], (_Float16)f[2 * e + 1]};
            o[e] = __builtin_bit_cast(unsigned, p);
        }
    }
    return o;
}
// f32 values as three bf16 parts, each what is left cut to 8 bits: together all 24.  An infinity is in its first part (what is left of it,
// NaN, becomes a number that its product does not notice)
__device__ __forceinline__ void cut3(const float (&x)[8], u32x4 (&part)[3]) {
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; e++) r[e] = x[e];
#pragma unroll
    for (int p = 0; p < 3; p++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const unsigned a = __float_as_uint(r[2 * e]) & 0xffff0000u, b = __float_as_uint(r[2 * e + 1]) & 0xffff0000u;
            part[p][e] = a >> 16 | b;
            r[2 * e] = fminf(fmaxf(r[2 * e] - __uint_as_float(a), -1e37f), 1e37f);
            r[2 * e + 1] = fminf(fmaxf(r[2 * e + 1] - __uint_as_float(b), -1e37f), 1e37f);
        }
}

// T: what the matrix cores take.  XF32: x is f32; else it is in PARTS arrays of T.  O: type of the scales and of y
template <class T, class O, bool XF32, int PARTS, bool GATE, int MT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) rows4_kernel(Rows4Args R) {
    constexpr int MATS = GATE ? 2 : 1, RUN = 128;
    __shared__ f32x4 sums[WAVES][MATS][MT][64];
    const int lane = threadIdx.x & 63, wave = TG_UNIFORM((int)(threadIdx.x >> 6)), i = lane & 15, q = lane >> 4;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * MT;
    // rows beyond the end repeat the last one: their results are not stored
    const uint8_t *codes[MATS];
    const O *scales[MATS][4];
    const char *x[MT];
#pragma unroll
    for (int a = 0; a < MATS; a++) {
        codes[a] = R.codes[a] + (size_t)min(n0 + i, R.N - 1) * R.ldc;
#pragma unroll
        for (int r = 0; r < 4; r++) scales[a][r] = (const O *)R.scales[a] + (size_t)min(n0 + 4 * q + r, R.N - 1) * R.lds;
    }
#pragma unroll
    for (int t = 0; t < MT; t++) x[t] = R.x + (size_t)min(m0 + 16 * t + i, R.M - 1) * R.ldx;
    f32x4 acc[MATS][MT];
#pragma unroll
    for (int a = 0; a < MATS; a++)
#pragma unroll
        for (int t = 0; t < MT; t++) acc[a][t] = f32x4{0, 0, 0, 0};
    const int steps = 1 << min(R.group_shift, 2);  // of 32 indices with one scale
    for (int k0 = wave * RUN; k0 < R.K; k0 += WAVES * RUN) {
        u32x4 w[MATS];
        const int kc = k0 + 32 * q;
#pragma unroll
        for (int a = 0; a < MATS; a++) w[a] = kc < R.K ? *(const u32x4 *)(codes[a] + kc / 2) : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int a = 0; a < MATS; a++) w[a] = exchange_words(w[a]);
        f32x4 sum[MATS][MT];
#pragma unroll
        for (int s = 0; s < 4; s++) {
            const int k = k0 + 32 * s + 8 * q;
            u32x4 f[MATS];
#pragma unroll
            for (int a = 0; a < MATS; a++) f[a] = codes8<T>(w[a][s]);
#pragma unroll
            for (int t = 0; t < MT; t++) {
                u32x4 b[PARTS];
                if constexpr (XF32) {
                    Oct<float> o;
                    get8((const float *)x[t] + k, R.K - k, o);
                    float v[8];
                    floats(o, v);
                    cut3(v, b);
                } else
#pragma unroll
                    for (int p = 0; p < PARTS; p++) b[p] = row_chunk<T>(x[t] + p * R.x_apart, k, R.K);
#pragma unroll
                for (int a = 0; a < MATS; a++) {
                    if (s % steps == 0) sum[a][t] = f32x4{0, 0, 0, 0};
#pragma unroll
                    for (int p = 0; p < PARTS; p++) sum[a][t] = mma<T>(f[a], b[p], sum[a][t]);
                }
            }
            if ((s + 1) % steps == 0 && k0 + 32 * s + 32 - 32 * steps < R.K) {
                const int g = (k0 + 32 * s) >> (5 + R.group_shift);
#pragma unroll
                for (int a = 0; a < MATS; a++)
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        const float scale = (float)scales[a][r][g];  // (times 16 it may be beyond f32)
#pragma unroll
                        for (int t = 0; t < MT; t++) acc[a][t][r] += scale * (16.0f * sum[a][t][r]);
                    }
            }
        }
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
    if constexpr (GATE) {
        float h[8];
#pragma unroll
        for (int e = 0; e < 8; e++) h[e] = n + e < R.N ? act_value(R.epi.act, v[0][e]) * v[1][e] : 0.0f;
        for (int p = 0; p < R.h_parts; p++) {
            store_oct((__bf16 *)R.h + p * R.h_apart + (size_t)m * R.ldh + n, h);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float part = (float)(__bf16)h[e];
                h[e] = fabsf(part) <= 3.4e38f ? h[e] - part : 0.0f;  // what is not finite is in its first part alone
            }
        }
    } else
        epilogue8<O, EPI_STORE>(R.epi, m, n, v[0], v[0]);
}

// ---- matrices to 4 bits and back: a wave takes a group of a row
struct Pack4Args {
    const char *w;
    char *w_out;
    uint8_t *codes;
    char *scales;
    size_t ldc, lds;  // bytes; elements
    int K, group;
    int64_t groups;   // of all rows
};
template <class W, class O> __global__ void __launch_bounds__(256) pack4_kernel(Pack4Args A) {
    const int lane = threadIdx.x & 63;
    const int64_t id = (int64_t)blockIdx.x * 4 + TG_UNIFORM((int)(threadIdx.x >> 6));
    if (id >= A.groups) return;
    const int64_t row = id / (int64_t)A.lds;
    const int k0 = (int)(id % (int64_t)A.lds) * A.group, end = min(k0 + A.group, A.K);
    const W *w = (const W *)A.w + (size_t)row * A.K;
    unsigned most = 0;  // word of the largest magnitude (NaN and infinity have the largest of all)
    for (int k = k0 + lane; k < end; k += 64) {
        const unsigned m = __float_as_uint((float)w[k]) & 0x7fffffffu;
        most = most > m ? most : m;
    }
    most = wave_max(most);
    float scale = (float)(O)(__uint_as_float(most) / 7.0f);
    const bool held = scale <= 3.4028234e38f;
    if (!held) scale = __uint_as_float(0x7fc00000u);
    const float inverse = held && scale > 0.0f ? 1.0f / scale : 0.0f;
    if (lane == 0) ((O *)A.scales)[id] = (O)scale;
    // 8 codes a lane, to the end of the row's 16 bytes
    const int stop = min(k0 + A.group, (A.K + 31) / 32 * 32);
    for (int k = k0 + 8 * lane; k < stop; k += 512) {
        unsigned c = 0;
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (k + e < A.K && inverse > 0.0f) c |= ((unsigned)(int)fminf(fmaxf(rintf((float)w[k + e] * inverse), -8.0f), 7.0f) & 15u) << (4 * e);
        *(unsigned *)(A.codes + (size_t)row * A.ldc + k / 2) = c;
    }
}
template <class W, class O> __global__ void __launch_bounds__(256) unpack4_kernel(Pack4Args A) {
    const int lane = threadIdx.x & 63;
    const int64_t id = (int64_t)blockIdx.x * 4 + TG_UNIFORM((int)(threadIdx.x >> 6));
    if (id >= A.groups) return;
    const int64_t row = id / (int64_t)A.lds;
    const int k0 = (int)(id % (int64_t)A.lds) * A.group, end = min(k0 + A.group, A.K);
    const float scale = (float)((const O *)A.scales)[id];
    for (int k = k0 + lane; k < end; k += 64)
        ((W *)A.w_out)[(size_t)row * A.K + k] = (W)(16.0f * code_to_float(A.codes[(size_t)row * A.ldc + k / 2] >> (k & 1 ? 4 : 0)) * scale);
}
