// Products of few rows with a matrix in 4 bits, y[m][o] = sum over groups G of scale[o][G] * (sum over k in G of code(o, k) x(m, k)): the codes
// are read once, 16 bytes a lane.
//
// A workgroup takes 16 rows of the matrix (GATE: 16 of each of two) and 16 * MT rows of x; its waves share the k axis in runs of 128.  Four
// lanes of a row read 32 codes each and exchange words, so that lane l holds what a step of the matrix cores takes of it: 8 codes of row l % 16
// from k0 + 32 s + 8 (l / 16) on for step s.  Codes become bf16 or f16 exactly (in sixteenths: that is what the
// conversion gives), a group's sum stays in f32 and is scaled there: a scaled weight rounded to 16 bits would cost three decimal
// places of four.  Sums stay in sixteenths to the end: 16 of a group's sum, or of its scale, may be beyond f32 where the answer is not.
// (Near f32's smallest numbers a group's product is rounded to 2^-146 of the answer so; products of single elements would be to 2^-150, 32 of them.)
// x: 16-bit as it is, f32 in three bf16 parts, cut as it is read; h between the block's products in two or three bf16 parts.
// The waves' sums meet in LDS and are added in their order.
// Bound by the codes' bytes (one row, 8192 -> 16384: 20 - 22.5 us, 3.1 - 3.4 TB/s), for small matrices by the latency of one trip to memory (1024 -> 4096,
// two of them: 7.4 us), and for many rows by x, which every workgroup of 16 columns reads and, in f32, cuts again (64 rows, 4096 -> 4096: 14.6 us in bf16,
// 26 - 29 in f32; workgroups of more columns would share it).  h in three parts for more than 32 rows takes two registers more than
// there are, with groups of 32 thirty-two (64 f32 rows of 1024 -> 4096 -> 1024: 40 us, with groups of 32 47)
#pragma once
#include "train_rows.h"

struct Rows4Args {
    const char *x;
    const uint8_t *codes[2];
    const char *scales[2];
    size_t ldx, ldc, lds;      // bytes; lds: elements of a row of scales
    size_t x_apart;            // bytes from one part of x to the next
    int M, N, K, group_shift;  // group = 32 << group_shift
    EpiArgs epi;
    char *h;                // GATE: act(g) u in bf16 parts, [parts][M][ldh]
    size_t ldh, h_apart;    // elements
    int h_parts;
};

#ifdef CKKSMI_EMULATE
#define code_to_float emu_code_to_float
#define exchange_words emu_exchange_words
#define wave_fence emu_wave_fence
#define TG_KEEP() (void)0
static inline unsigned upper_halves(float low, float high) { return __float_as_uint(low) >> 16 | (__float_as_uint(high) & 0xffff0000u); }
static inline float within(float x, float most) { return fminf(fmaxf(x, -most), most); }
static inline float quieted(float x) { return x == x ? x : __uint_as_float(__float_as_uint(x) | 0x400000u); }
#else
// what the wave wrote to LDS is there for all of its lanes (a wave's LDS instructions keep their order)
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
#define TG_KEEP() asm volatile("" ::: "memory")  // loads before it stay before it (the compiler would move those of a later round to their use)
__device__ __forceinline__ unsigned upper_halves(float low, float high) { return __builtin_amdgcn_perm(__float_as_uint(high), __float_as_uint(low), 0x07060302u); }
__device__ __forceinline__ float within(float x, float most) { return __builtin_amdgcn_fmed3f(x, -most, most); }  // (of NaN: a number)
__device__ __forceinline__ float quieted(float x) { return __builtin_canonicalizef(x); }  // (a NaN gets its quiet bit: one in the upper half of its word)
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

// f32 x is read in two pieces of 4 indices a lane, 16 apart, so that the lanes of a row read 64 bytes in a row: word j of the result has the codes of
// indices 4 j .. + 3 and 16 + 4 j .. + 3
__device__ __forceinline__ u32x4 halves_apart(u32x4 w) {
    return u32x4{(w[0] & 0xffffu) | w[2] << 16, w[0] >> 16 | (w[2] & 0xffff0000u), (w[1] & 0xffffu) | w[3] << 16, w[1] >> 16 | (w[3] & 0xffff0000u)};
}

// 8 codes as T, in sixteenths
template <class T> __device__ __forceinline__ u32x4 codes8(unsigned w) {
    unsigned v = w >> 4;
    TG_OPAQUE(v);
    float f[8];
#pragma unroll
    for (int e = 0; e < 4; e++) {  // (bytes, which the conversion selects by itself)
        f[2 * e] = code_to_float(w >> (8 * e) & 0xffu);
        f[2 * e + 1] = code_to_float(v >> (8 * e) & 0xffu);
    }
    u32x4 o;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        if constexpr (__is_same(T, __bf16)) o[e] = upper_halves(f[2 * e], f[2 * e + 1]);
        else {
            struct { _Float16 low, high; } p = {(_Float16)f[2 * e], (_Float16)f[2 * e + 1]};
            o[e] = __builtin_bit_cast(unsigned, p);
        }
    }
    return o;
}
// f32 values as three bf16 parts, each what is left cut to 8 bits: together all 24 (to bf16's smallest number, 2^-133).  An infinity is in its first part
// (what is left of it, NaN, becomes a number that its product does not notice), and so is a NaN: cut as it is, one whose payload
// lies in the lower half of its word would be an infinity
__device__ __forceinline__ void cut3(const float (&x)[8], u32x4 (&part)[3]) {
#pragma unroll
    for (int e = 0; e < 4; e++) {
        float r[2] = {quieted(x[2 * e]), quieted(x[2 * e + 1])};
#pragma unroll
        for (int p = 0; p < 3; p++) {
            part[p][e] = upper_halves(r[0], r[1]);
#pragma unroll
            for (int k = 0; k < 2; k++) {
                r[k] -= __uint_as_float(__float_as_uint(r[k]) & 0xffff0000u);
                if (p == 0) r[k] = within(r[k], 1e37f);
            }
        }
    }
}

// T: what the matrix cores take.  XF32: x is f32; else it is in PARTS arrays of T.  O: type of the scales and of y.  EACH: steps of 32 indices that
// have a scale of their own (1, 2; 4: the scale is the run's)
template <class T, class O, bool XF32, int PARTS, bool GATE, int MT, int WAVES, int EACH>
__global__ void __launch_bounds__(64 * WAVES) rows4_kernel(Rows4Args R) {
    constexpr int MATS = GATE ? 2 : 1, RUN = 128, WORDS = XF32 ? 2 : PARTS;
    // a wave's own: what its lanes exchange, in the end its sums
    constexpr int AREA = MATS * MT > MT * WORDS ? MATS * MT : MT * WORDS;
    __shared__ u32x4 areas[WAVES][AREA][64];
    __shared__ __attribute__((aligned(16))) float scale_slots[WAVES][MATS][64];
    const int lane = threadIdx.x & 63, wave = TG_UNIFORM((int)(threadIdx.x >> 6)), i = lane & 15, q = lane >> 4;
    u32x4(*const area)[64] = areas[wave];
    // Neighbouring lanes read neighbouring memory: lane l 16 bytes of row l / 4, piece l % 4 (16 lanes of 16 rows would keep the memory path
    // busy four times as long); through LDS they come to lane l % 16 + 16 * piece, which the matrix cores take them from.  The pieces of
    // a row lie in another order every four rows, so that the lanes that read together spread over the banks
    const int row = lane >> 2, piece = lane & 3, to = (lane & ~3) | (piece ^ (row >> 2)), from = 4 * i + (q ^ (i >> 2));
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * MT;
    // rows beyond the end repeat the last one (of the matrix) or are zeros (of x): their results are not stored.  Addresses are a scalar and a
    // lane's 32-bit offset, which stays the same along k
    const uint8_t *codes[MATS];
    const O *scales[MATS];
    const char *x[MT];
    const unsigned n_row = min(row, R.N - 1 - n0), code_offset = n_row * (unsigned)R.ldc + 16 * piece, x_offset = row * (unsigned)R.ldx;
    const unsigned scale_offset = n_row * (unsigned)R.lds + (piece >> R.group_shift);
#pragma unroll
    for (int a = 0; a < MATS; a++) {
        codes[a] = R.codes[a] + (size_t)n0 * R.ldc;
        scales[a] = (const O *)R.scales[a] + (size_t)n0 * R.lds;
    }
#pragma unroll
    for (int t = 0; t < MT; t++) x[t] = R.x + (size_t)(m0 + 16 * t) * R.ldx;
    f32x4 acc[MATS][MT];
#pragma unroll
    for (int a = 0; a < MATS; a++)
#pragma unroll
        for (int t = 0; t < MT; t++) acc[a][t] = f32x4{0, 0, 0, 0};

    // Lanes request what somebody needs and no more: x of rows that there are, a scale once a group.
    // A run's codes (32 indices a piece) and scales; x of a step of 32 indices
    struct Codes { u32x4 w[MATS]; O s[MATS]; };
    struct X { u32x4 v[MT][WORDS]; };
    constexpr int STEPS = MT * WORDS <= 2 ? 4 : MT * WORDS <= 4 ? 2 : 1;  // of x that are requested together
    auto load_codes = [&](Codes &c, int k0) {
#pragma unroll
        for (int a = 0; a < MATS; a++) {
            c.w[a] = *(const u32x4 *)(codes[a] + k0 / 2 + code_offset);
            if (piece % EACH == 0) c.s[a] = (scales[a] + (k0 >> (5 + R.group_shift)))[scale_offset];
        }
    };
    // f32: pieces of 4 indices, two of them 16 apart; else of 8 in each part
    auto load_x = [&](X &b, int k) {
#pragma unroll
        for (int t = 0; t < MT; t++) {
            if (m0 + 16 * t + row >= R.M) continue;
#pragma unroll
            for (int p = 0; p < WORDS; p++)
                __builtin_memcpy(&b.v[t][p], (XF32 ? x[t] + (size_t)(k + 16 * p) * 4 : x[t] + p * R.x_apart + (size_t)k * 2) + (x_offset + 16 * piece), 16);
        }
    };
    // a run's products; x_of(s): x of step s
    auto take = [&](const Codes &c, auto x_of) {
        u32x4 w[MATS];
        wave_fence();
#pragma unroll
        for (int a = 0; a < MATS; a++) {
            area[a][to] = XF32 ? halves_apart(c.w[a]) : c.w[a];
            scale_slots[wave][a][16 * piece + row] = (float)c.s[a];
        }
        wave_fence();
#pragma unroll
        for (int a = 0; a < MATS; a++) w[a] = exchange_words(area[a][from]);
        f32x4 sum[MATS][MT];
#pragma unroll
        for (int s = 0; s < 4; s++) {
            X now = x_of(s);
            wave_fence();
#pragma unroll
            for (int t = 0; t < MT; t++)
#pragma unroll
                for (int p = 0; p < WORDS; p++) area[t * WORDS + p][to] = now.v[t][p];
            wave_fence();
            u32x4 f[MATS];
#pragma unroll
            for (int a = 0; a < MATS; a++) f[a] = codes8<T>(w[a][s]);
#pragma unroll
            for (int t = 0; t < MT; t++) {
                u32x4 part[PARTS];
                if constexpr (XF32) {
                    float v[8];
#pragma unroll
                    for (int p = 0; p < 2; p++) __builtin_memcpy(v + 4 * p, &area[t * WORDS + p][from], 16);
                    cut3(v, part);
                } else
#pragma unroll
                    for (int p = 0; p < PARTS; p++) part[p] = area[t * WORDS + p][from];
#pragma unroll
                for (int a = 0; a < MATS; a++) {
                    if (s % EACH == 0) sum[a][t] = f32x4{0, 0, 0, 0};
#pragma unroll
                    for (int p = 0; p < PARTS; p++) sum[a][t] = mma<T>(f[a], part[p], sum[a][t]);
                }
            }
            if ((s + 1) % EACH == 0)
#pragma unroll
                for (int a = 0; a < MATS; a++) {
                    const f32x4 scale = *(const f32x4 *)&scale_slots[wave][a][16 * (s + 1 - EACH) + 4 * q];  // of rows 4 (l / 16) .. + 3
#pragma unroll
                    for (int t = 0; t < MT; t++)
#pragma unroll
                        for (int r = 0; r < 4; r++) acc[a][t][r] = fmaf(scale[r], sum[a][t][r], acc[a][t][r]);
                }
        }
    };
    // Whole runs: nothing in the way of the loads that are under way.  A run's codes, scales and first steps of x are requested before the run before
    // it is taken, into one of two sets of registers (one set that is copied would be waited for)
    const int whole = R.K / RUN;
    struct Ahead { Codes c; X x[STEPS]; };
    auto request = [&](Ahead &h, int run) {
        load_codes(h.c, run * RUN);
#pragma unroll
        for (int s = 0; s < STEPS; s++) load_x(h.x[s], run * RUN + 32 * s);
    };
    auto take_run = [&](Ahead &h, int run) {
        TG_SCHEDULED();
        take(h.c, [&](int s) {
            const X v = h.x[s % STEPS];
            if (s + STEPS < 4) load_x(h.x[s % STEPS], run * RUN + 32 * (s + STEPS));
            return v;
        });
        TG_KEEP();
    };
    const int second = whole >= 2 * WAVES ? 1 : WAVES, begin = second == 1 ? 2 * wave : wave;  // pairs of runs share 128 bytes of a row
    if (begin < whole) {
        Ahead h[2] = {};  // (lanes that request nothing keep zeros)
        request(h[0], begin);
        for (int run = begin; run < whole; run += 2 * WAVES) {
            request(h[1], min(run + second, whole - 1));  // (the last time to no purpose)
            take_run(h[0], run);
            if (run + second >= whole) break;
            request(h[0], min(run + 2 * WAVES, whole - 1));
            take_run(h[1], run + second);
        }
    }
    // the last indices, if they are no whole run: zeros behind them (a group that lies behind them has sums 0 and scale 0)
    if (R.K % RUN && wave == whole % WAVES) {
        const int k0 = whole * RUN, k = k0 + 32 * piece;
        Codes c;
#pragma unroll
        for (int a = 0; a < MATS; a++) {
            c.w[a] = u32x4{0, 0, 0, 0};
            c.s[a] = (O)0.0f;
            if (k < R.K) {
                c.w[a] = *(const u32x4 *)(codes[a] + k0 / 2 + code_offset);
                c.s[a] = (scales[a] + (k0 >> (5 + R.group_shift)))[scale_offset];
            }
        }
        take(c, [&](int s) {
            X v{};
            const int ks = k0 + 32 * s;
#pragma unroll
            for (int t = 0; t < MT; t++) {
                if (m0 + 16 * t + row >= R.M) continue;
#pragma unroll
                for (int p = 0; p < WORDS; p++)
                    if constexpr (XF32) v.v[t][p] = row_chunk<float>(x[t] + x_offset, ks + 16 * p + 4 * piece, R.K);
                    else v.v[t][p] = row_chunk<T>(x[t] + x_offset + p * R.x_apart, ks + 8 * piece, R.K);
            }
            return v;
        });
    }
    wave_fence();
#pragma unroll
    for (int a = 0; a < MATS; a++)
#pragma unroll
        for (int t = 0; t < MT; t++) __builtin_memcpy(&area[a * MT + t][lane], &acc[a][t], 16);
    __syncthreads();
    auto sums_of = [&](int wave, int a, int t, int lane) {
        f32x4 s;
        __builtin_memcpy(&s, &areas[wave][a * MT + t][lane], 16);
        return s;
    };
    // lane l's sums are row l % 16's columns 4*(l/16) .. +3: a thread takes 8 columns of a row
    if (threadIdx.x >= 32 * MT) return;
    const int t = threadIdx.x / 32, r = threadIdx.x % 16, half = threadIdx.x / 16 % 2, m = m0 + 16 * t + r, n = n0 + 8 * half;
    if (m >= R.M || n >= R.N) return;
    float v[2][8];
#pragma unroll
    for (int a = 0; a < MATS; a++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
            f32x4 s = sums_of(0, a, t, (2 * half + e) * 16 + r);
#pragma unroll 3
            for (int k = 1; k < WAVES; k++) s += sums_of(k, a, t, (2 * half + e) * 16 + r);
#pragma unroll
            for (int j = 0; j < 4; j++) v[a][4 * e + j] = 16.0f * s[j];
        }
    if constexpr (GATE) {
        float h[8];
#pragma unroll
        for (int e = 0; e < 8; e++) h[e] = n + e < R.N ? act_value(R.epi.act, v[0][e]) * v[1][e] : 0.0f;
        for (int p = 0; p < R.h_parts; p++) {
            // (a part is at most bf16's largest number, 3.3895e38: rounded, a finite h beyond it would be an infinity)
            float part[8];
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const bool finite = fabsf(h[e]) <= 3.4028235e38f;
                part[e] = finite ? (float)(__bf16)within(h[e], 3.3895314e38f) : h[e];
                h[e] = finite ? h[e] - part[e] : 0.0f;  // what is not finite is in its first part alone
            }
            store_oct((__bf16 *)R.h + p * R.h_apart + (size_t)m * R.ldh + n, part);
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
    if (lane == 0) ((O *)A.scales)[id] = (O)scale;
    // 8 codes a lane, to the end of the row's 16 bytes
    const int stop = min(k0 + A.group, (A.K + 31) / 32 * 32);
    for (int k = k0 + 8 * lane; k < stop; k += 512) {
        unsigned c = 0;
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (k + e < A.K && scale > 0.0f) c |= ((unsigned)(int)fminf(fmaxf(rintf((float)w[k + e] / scale), -8.0f), 7.0f) & 15u) << (4 * e);  // (1 / scale may be beyond f32)
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
