// Norms before and after a block with its gate and residual sum: r = a x + b gate N1(f), n = N2(r), and their backward pass.
//
// A row's norm needs all of the row before its first result: a group of threads holds a row in registers, 8 neighbouring elements a thread (16
// for forward rows beyond 8192), so every operand is read once, and the columns' weights once per group.  Layer norms of the widest rows
// do not fit the 128 registers of a thread of 1024 and keep some in memory: 19 - 29 forward beyond 8192, 153 - 201 backward beyond 4096 (with the
// columns' sums and weights), where both passes take 293 us for 4096 bf16 rows of 8192, of rms norms 180.  With h = (v - mean) s, s = 1 / sqrt(mean (v - mean)^2 + eps),
// the gradient of N(v) = h w + b by v is, for g = dy w,
//     dv = (g - mean(g) - h mean(g h)) s          (rms: without the first mean)
// The forward pass saves each row's two means and two s; the backward pass forms h of both norms again from x and f and needs two rounds of sums
// over the row.  Sums over rows: a thread keeps up to four for each of its columns over all rows that its group takes,
//     P = sum of dy h1, Q = sum of dy (dy: gradient of N1(f), without a channel's gate), R = sum of dn h2, T = sum of dn,
// workgroups' sums go to memory once, and a second kernel adds them in their order: gradients of w1, b1, w2, b2 are P g, Q g, R, T, and of a
// channel's gate g it is P w1 + Q b1.
// A norm that is not there has mean 0, s 1, w 1 and b 0; a block that is not there f = 0, a = 1, b = 0: the same results without a case.
// Longer rows than registers hold (forward beyond 16384, backward beyond 8192) are read once for each sum; their column sums take a pass of their
// own: 2048 bf16 rows of 16384, rms, both passes, 364 us (1.85 TB/s of what they need); 1024 rows of 65536, forward, 234 us (2.3).
// Bound by memory: 4096 f32 rows of 4096, forward, 48 - 57 us, 4.6 TB/s and more (a large copy: 4.7); 16384 bf16 rows of 2048 60 us forward (4.5), 109
// backward (3.7: six operands, and 512 or 768 workgroups whose last rows end at different times); with layer norms both 225; one row 3.7 us, a
// launch
#pragma once
#include "train_types.h"

struct NormArgs {
    const char *x, *f, *gate;
    const char *post_w, *post_b, *pre_w, *pre_b;
    char *r, *n;
    float *stats;  // [rows][4]: mean and s of f, of r
    const char *dr, *dn;
    char *dx, *df, *dgate;
    float *part;   // [workgroups][vectors][ld_part]
    float *coef;   // long rows: [rows][4]: mean(g), mean(g h) of n's norm, of f's
    size_t ld_x, ld_f, ld_gate, ld_r, ld_n, ld_dr, ld_dn, ld_dx, ld_df, ld_dgate;  // bytes
    size_t ld_part;
    int M, d;
    int pre, post, gate_kind;  // CKKSMI_*
    int w_f32;                 // the weights are f32 whatever the rows
    int sums;                  // bits of enum NormSum: column sums that are wanted
    int vectors;               // their number
    float eps, a, b, inv_d;
};
// column sums, in the order in which they lie in NormArgs::part
enum NormSum { SUM_P = 1, SUM_Q = 2, SUM_R = 4, SUM_T = 8, NORM_SUMS = 4 };

// 8 elements to p, of which `left` exist
template <class T> __device__ __forceinline__ void put8(T *p, int left, const float (&x)[8]) {
    Oct<T> o;
#pragma unroll
    for (int e = 0; e < 8; e++) o.v[e] = (T)x[e];
    if (left >= 8) __builtin_memcpy(p, &o, sizeof(o));
    else
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (e < left) p[e] = o.v[e];
}
// 8 values of a weight, a bias or a channel gate; `missing` where there is none
template <class T> __device__ __forceinline__ void weights8(const char *w, int w_f32, int at, int left, float missing, float (&x)[8]) {
    if (!w)
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] = missing;
    else if (w_f32 || sizeof(T) == 4) {
        Oct<float> o;
        get8((const float *)w + at, left, o);
        floats(o, x);
    } else {
        Oct<T> o;
        get8((const T *)w + at, left, o);
        floats(o, x);
    }
}

// ---- sums over a row's group of threads; every thread gets the same bits (pairs are added in the same order on both sides)
#ifdef CKKSMI_EMULATE
template <int LANES> static inline float lanes_sum(float x) { return emu_lanes_sum(x, LANES); }
#else
template <int CONTROL> __device__ __forceinline__ float add_dpp(float x) {
    return x + __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CONTROL, 0xf, 0xf, true));
}
// neighbours, pairs, halves of 8, halves of 16, then rows of 16 lanes and halves of the wave
template <int LANES> __device__ __forceinline__ float lanes_sum(float x) {
    x = add_dpp<0xB1>(x);
    x = add_dpp<0x4E>(x);
    x = add_dpp<0x141>(x);
    if constexpr (LANES >= 16) x = add_dpp<0x140>(x);
    if constexpr (LANES >= 32) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    if constexpr (LANES >= 64) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return x;
}
#endif

// LANES threads sum two values; more than a wave meet in LDS.  (Two sets of slots: a set is written again only after everyone has come
// past the other set's barrier, hence has read it)
template <int LANES> struct RowSums {
    static constexpr int WAVES = LANES > 64 ? LANES / 64 : 1;
    float (*slots)[WAVES][2];
    int phase = 0;
    __device__ __forceinline__ explicit RowSums(float (*s)[WAVES][2]) : slots(s) {}
    __device__ __forceinline__ void operator()(float &a, float &b) {
        constexpr int IN_WAVE = LANES > 64 ? 64 : LANES;
        a = lanes_sum<IN_WAVE>(a);
        b = lanes_sum<IN_WAVE>(b);
        if constexpr (WAVES > 1) {
            float(*s)[2] = slots[phase];
            phase ^= 1;
            if ((threadIdx.x & 63) == 0) {
                s[threadIdx.x >> 6][0] = a;
                s[threadIdx.x >> 6][1] = b;
            }
            __syncthreads();
            a = s[0][0];
            b = s[0][1];
#pragma unroll
            for (int w = 1; w < WAVES; w++) {
                a += s[w][0];
                b += s[w][1];
            }
        }
    }
    __device__ __forceinline__ void operator()(float &a) {
        float b = 0.0f;
        (*this)(a, b);
    }
};

// A layer norm's mean is a sum in 32 bits, some last places off: of a row of equal numbers, 1e4 say, what is left of them would be normed to 0.3 and more.
// The sum of what is left says how far it is off, and with it comes the sum of squares: q of the mean before, t that sum
__device__ __forceinline__ void right_mean(const NormArgs &A, float t, float &mean, float &q) {
    const float by = t * A.inv_d;
    mean += by;
    q = fmaxf(fmaf(-t, by, q), 0.0f);  // (a row that is not finite has a mean that is not)
}

// mean and s of a row's values that the group holds (elements beyond the row are zeros)
template <bool LAYER, int LANES, int V>
__device__ __forceinline__ void row_stats(const NormArgs &A, int kind, int t, const float (&v)[V][8], RowSums<LANES> &sums, float &mean, float &s) {
    mean = 0.0f;
    if (LAYER && kind == CKKSMI_NORM_LAYER) {
#pragma unroll
        for (int j = 0; j < V; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) mean += v[j][e];
        sums(mean);
        mean *= A.inv_d;
    }
    float q = 0.0f, left = 0.0f;
#pragma unroll
    for (int j = 0; j < V; j++)
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float c = LAYER ? (8 * (t + LANES * j) + e < A.d ? v[j][e] - mean : 0.0f) : v[j][e];
            q = fmaf(c, c, q);
            if (LAYER) left += c;
        }
    if (LAYER && kind == CKKSMI_NORM_LAYER) {
        sums(q, left);
        right_mean(A, left, mean, q);
    } else
        sums(q);
    s = 1.0f / sqrtf(q * A.inv_d + A.eps);
}

// Weights of 8 columns: of N1, the gate (a channel's), of N2
struct NormWeights { float w1[8], b1[8], g[8], w2[8], b2[8]; };
template <class T, bool LAYER> __device__ __forceinline__ void norm_weights(const NormArgs &A, int at, NormWeights &w) {
    const int left = A.d - at;
    weights8<T>(A.post_w, A.w_f32, at, left, 1.0f, w.w1);
    weights8<T>(A.gate_kind == CKKSMI_GATE_CHANNEL ? A.gate : nullptr, A.w_f32, at, left, 1.0f, w.g);
    weights8<T>(A.pre_w, A.w_f32, at, left, 1.0f, w.w2);
    if (LAYER) {
        weights8<T>(A.post_b, A.w_f32, at, left, 0.0f, w.b1);
        weights8<T>(A.pre_b, A.w_f32, at, left, 0.0f, w.b2);
    }
}
// h of N1, N1(f), and r
template <bool LAYER>
__device__ __forceinline__ float norm_sum(const NormArgs &A, const NormWeights &w, int e, float x, float f, float g, float mean1, float s1, float &h1, float &y) {
    h1 = LAYER ? (f - mean1) * s1 : f * s1;
    y = LAYER ? fmaf(h1, w.w1[e], w.b1[e]) : h1 * w.w1[e];
    return fmaf(A.b, y * g, A.a * x);
}

// Rows are taken by groups of LANES threads, 8 * V * LANES elements at most each; GROUPS of them in a workgroup
template <int LANES> struct NormShape {
    static constexpr int THREADS = LANES > 64 ? LANES : 256, GROUPS = THREADS / LANES;
    // (a row's index is a scalar where a group has whole waves)
    static __device__ __forceinline__ int group() { return GROUPS == 1 ? 0 : LANES == 64 ? TG_UNIFORM((int)(threadIdx.x / LANES)) : (int)(threadIdx.x / LANES); }
    static __device__ __forceinline__ int lane() { return GROUPS == 1 ? (int)threadIdx.x : (int)(threadIdx.x % LANES); }
};

template <class T, int LANES, int V, bool LAYER>
__global__ void __launch_bounds__(NormShape<LANES>::THREADS) norm_forward_kernel(NormArgs A) {
    constexpr int GROUPS = NormShape<LANES>::GROUPS;
    __shared__ float slots[2][RowSums<LANES>::WAVES][2];
    RowSums<LANES> sums(slots);
    const int t = NormShape<LANES>::lane(), group = NormShape<LANES>::group();
    struct Row { Oct<T> x[V], f[V], g[V]; };
    auto load = [&](Row &w, int row_) {
        const size_t row = row_;
#pragma unroll
        for (int j = 0; j < V; j++) {
            const int at = 8 * (t + LANES * j), left = A.d - at;
            w.f[j] = Oct<T>{};
            get8((const T *)(A.x + row * A.ld_x) + at, left, w.x[j]);
            if (A.f) get8((const T *)(A.f + row * A.ld_f) + at, left, w.f[j]);
            if (A.gate_kind == CKKSMI_GATE_ELEMENT) get8((const T *)(A.gate + row * A.ld_gate) + at, left, w.g[j]);
        }
    };
    Row next;
    const int stride = gridDim.x * GROUPS;
    load(next, min((int)blockIdx.x * GROUPS + group, A.M - 1));
    NormWeights kept;  // (two of them would leave no registers for the rows)
    if (V == 1) norm_weights<T, LAYER>(A, 8 * t, kept);
    for (int first = blockIdx.x * GROUPS; first < A.M; first += stride) {
        // (a group without a row repeats the last one and stores nothing)
        const int row = min(first + group, A.M - 1);
        const bool mine = first + group < A.M;
        const Row now = next;
        load(next, first < A.M - stride ? min(first + stride + group, A.M - 1) : row);  // (the last time: to no purpose)
        float v[V][8];
        float mean1 = 0.0f, s1 = 1.0f, mean2 = 0.0f, s2 = 1.0f;
#pragma unroll
        for (int j = 0; j < V; j++) floats(now.f[j], v[j]);
        if (A.post != CKKSMI_NORM_NONE) row_stats<LAYER, LANES, V>(A, A.post, t, v, sums, mean1, s1);
#pragma unroll
        for (int j = 0; j < V; j++) {
            const int at = 8 * (t + LANES * j);
            NormWeights other;
            if (V > 1) norm_weights<T, LAYER>(A, at, other);
            const NormWeights &w = V > 1 ? other : kept;
            float x[8], g[8], h, y;
            floats(now.x[j], x);
            if (A.gate_kind == CKKSMI_GATE_ELEMENT) floats(now.g[j], g);
            else
#pragma unroll
                for (int e = 0; e < 8; e++) g[e] = w.g[e];
#pragma unroll
            for (int e = 0; e < 8; e++) {
                v[j][e] = norm_sum<LAYER>(A, w, e, x[e], v[j][e], g[e], mean1, s1, h, y);
                if (LAYER && at + e >= A.d) v[j][e] = 0.0f;  // (without means it is 0 there)
            }
            if (A.r && mine) put8((T *)(A.r + (size_t)row * A.ld_r) + at, A.d - at, v[j]);
        }
        if (A.pre != CKKSMI_NORM_NONE) {
            row_stats<LAYER, LANES, V>(A, A.pre, t, v, sums, mean2, s2);
#pragma unroll
            for (int j = 0; j < V; j++) {
                const int at = 8 * (t + LANES * j);
                NormWeights other;
                if (V > 1) norm_weights<T, LAYER>(A, at, other);
                const NormWeights &w = V > 1 ? other : kept;
#pragma unroll
                for (int e = 0; e < 8; e++) v[j][e] = LAYER ? fmaf((v[j][e] - mean2) * s2, w.w2[e], w.b2[e]) : v[j][e] * s2 * w.w2[e];
                if (mine) put8((T *)(A.n + (size_t)row * A.ld_n) + at, A.d - at, v[j]);
            }
        }
        if (A.stats && mine && t == 0) *(f32x4 *)(A.stats + 4 * (size_t)row) = f32x4{mean1, s1, mean2, s2};
    }
}

// 8 elements of a row on their way back: h of both norms, N1(f), an element's gate, the gradients of r and n
struct NormBack { float h1[8], y[8], g[8], h2[8], dt[8], dn[8]; };
template <class T, bool LAYER, bool ELEMENT>
__device__ __forceinline__ void back_begin(const NormArgs &A, const NormWeights &w, const Oct<T> &ox, const Oct<T> &of, const Oct<T> &og, const Oct<T> &odr, const Oct<T> &odn,
                                           const f32x4 &st, NormBack &B) {
    float x[8], f[8];
    floats(ox, x);
    floats(of, f);
    floats(odr, B.dt);
    floats(odn, B.dn);
    if (ELEMENT) floats(og, B.g);
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const float r = norm_sum<LAYER>(A, w, e, x[e], f[e], ELEMENT ? B.g[e] : w.g[e], st[0], st[1], B.h1[e], B.y[e]);
        B.h2[e] = LAYER ? (r - st[2]) * st[3] : r * st[3];
    }
}
// shares of mean(g), mean(g h) of n's norm, and (below) of f's.  (Beyond the row all of g is 0; h is not where there are means, but finite
// unless the row is not)
template <bool LAYER> __device__ __forceinline__ void back_pre_sums(const NormArgs &A, const NormWeights &w, const NormBack &B, int left, float &s0, float &s1) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const float g = B.dn[e] * w.w2[e];
        if (LAYER) s0 += g;
        s1 = LAYER && e >= left ? s1 : fmaf(g, B.h2[e], s1);
    }
}
// dt: the gradient of r
template <bool LAYER> __device__ __forceinline__ void back_r(const NormArgs &A, const NormWeights &w, NormBack &B, const f32x4 &st, float m0, float m1) {
    if (A.pre == CKKSMI_NORM_NONE) return;
#pragma unroll
    for (int e = 0; e < 8; e++) B.dt[e] = fmaf(fmaf(-B.h2[e], m1, LAYER ? B.dn[e] * w.w2[e] - m0 : B.dn[e] * w.w2[e]), st[3], B.dt[e]);
}
// gradient of N1(f) without a channel's gate, and of h1
template <bool ELEMENT> __device__ __forceinline__ float back_y(const NormArgs &A, const NormBack &B, int e) { return ELEMENT ? B.dt[e] * A.b * B.g[e] : B.dt[e] * A.b; }
template <bool ELEMENT> __device__ __forceinline__ float back_h(const NormArgs &A, const NormWeights &w, const NormBack &B, int e) {
    return back_y<ELEMENT>(A, B, e) * (ELEMENT ? w.w1[e] : w.g[e] * w.w1[e]);
}
template <bool LAYER, bool ELEMENT> __device__ __forceinline__ void back_post_sums(const NormArgs &A, const NormWeights &w, const NormBack &B, int left, float &s0, float &s1) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const float g = LAYER && e >= left ? 0.0f : back_h<ELEMENT>(A, w, B, e);
        if (LAYER) s0 += g;
        s1 = LAYER && e >= left ? s1 : fmaf(g, B.h1[e], s1);
    }
}
// gradients of the elements to memory
template <class T, bool LAYER, bool ELEMENT>
__device__ __forceinline__ void back_store(const NormArgs &A, const NormWeights &w, int at, size_t row, const NormBack &B, const f32x4 &st, float m0, float m1) {
    const int left = A.d - at;
    float o[8];
    if (A.dx) {
#pragma unroll
        for (int e = 0; e < 8; e++) o[e] = B.dt[e] * A.a;
        put8((T *)(A.dx + row * A.ld_dx) + at, left, o);
    }
    if (ELEMENT && A.dgate) {
#pragma unroll
        for (int e = 0; e < 8; e++) o[e] = B.dt[e] * A.b * B.y[e];
        put8((T *)(A.dgate + row * A.ld_dgate) + at, left, o);
    }
    if (A.df) {
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float g = back_h<ELEMENT>(A, w, B, e);
            o[e] = A.post == CKKSMI_NORM_NONE ? g : fmaf(-B.h1[e], m1, LAYER ? g - m0 : g) * st[1];
        }
        put8((T *)(A.df + row * A.ld_df) + at, left, o);
    }
}
// a row's terms of the column sums
template <bool LAYER, bool ELEMENT> __device__ __forceinline__ void back_columns(const NormArgs &A, const NormBack &B, float (&sum)[NORM_SUMS][8]) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const float dy = back_y<ELEMENT>(A, B, e);
        sum[0][e] = fmaf(dy, B.h1[e], sum[0][e]);
        if (LAYER) sum[1][e] += dy;
        sum[2][e] = fmaf(B.dn[e], B.h2[e], sum[2][e]);
        if (LAYER) sum[3][e] += B.dn[e];
    }
}
// column sums of a workgroup (of a wave, for long rows) to memory
__device__ __forceinline__ void put_columns(const NormArgs &A, size_t group, int at, const float (&sum)[NORM_SUMS][8]) {
    float *p = A.part + group * A.vectors * A.ld_part + at;
#pragma unroll
    for (int k = 0; k < NORM_SUMS; k++)
        if (A.sums >> k & 1) {
            if (at < A.d) store_oct(p, sum[k]);
            p += A.ld_part;
        }
}

template <class T, int LANES, bool LAYER, bool ELEMENT>
__global__ void __launch_bounds__(NormShape<LANES>::THREADS) norm_backward_kernel(NormArgs A) {
    constexpr int GROUPS = NormShape<LANES>::GROUPS;
    __shared__ float slots[2][RowSums<LANES>::WAVES][2];
    RowSums<LANES> sums(slots);
    const int t = NormShape<LANES>::lane(), group = NormShape<LANES>::group(), at = 8 * t, left = A.d - at;
    struct Row { Oct<T> x, f, g, dr, dn; f32x4 st; };
    auto load = [&](Row &w, int row_) {
        const size_t row = row_;
        w.st = *(const f32x4 *)(A.stats + 4 * row);
        w.f = w.dr = w.dn = Oct<T>{};
        get8((const T *)(A.x + row * A.ld_x) + at, left, w.x);
        if (A.f) get8((const T *)(A.f + row * A.ld_f) + at, left, w.f);
        if (ELEMENT) get8((const T *)(A.gate + row * A.ld_gate) + at, left, w.g);
        if (A.dr) get8((const T *)(A.dr + row * A.ld_dr) + at, left, w.dr);
        if (A.dn) get8((const T *)(A.dn + row * A.ld_dn) + at, left, w.dn);
    };
    // the next row is on its way while one is computed; of wide rows two workgroups a compute unit have other rows on their way instead (8192 rows
    // of 4096: 166 us both passes, with one workgroup and the next row 209)
    constexpr bool AHEAD = LANES < 512;
    Row next;
    const int stride = gridDim.x * GROUPS;
    if (AHEAD) load(next, min((int)blockIdx.x * GROUPS + group, A.M - 1));
    NormWeights w;
    norm_weights<T, LAYER>(A, at, w);
    float columns[NORM_SUMS][8];
#pragma unroll
    for (int k = 0; k < NORM_SUMS; k++)
#pragma unroll
        for (int e = 0; e < 8; e++) columns[k][e] = 0.0f;
    for (int first = blockIdx.x * GROUPS; first < A.M; first += stride) {
        const int row = min(first + group, A.M - 1);
        const bool mine = first + group < A.M;
        Row now;
        if (AHEAD) now = next;
        else load(now, row);
        if (AHEAD) load(next, first < A.M - stride ? min(first + stride + group, A.M - 1) : row);  // (the last time: to no purpose)
        NormBack B;
        back_begin<T, LAYER, ELEMENT>(A, w, now.x, now.f, now.g, now.dr, now.dn, now.st, B);
        float m0 = 0.0f, m1 = 0.0f;
        if (A.pre != CKKSMI_NORM_NONE) {
            back_pre_sums<LAYER>(A, w, B, left, m0, m1);
            sums(m0, m1);
            m0 = A.pre == CKKSMI_NORM_LAYER ? m0 * A.inv_d : 0.0f;
            m1 *= A.inv_d;
            back_r<LAYER>(A, w, B, now.st, m0, m1);
        }
        m0 = m1 = 0.0f;
        if (A.post != CKKSMI_NORM_NONE) {
            back_post_sums<LAYER, ELEMENT>(A, w, B, left, m0, m1);
            sums(m0, m1);
            m0 = A.post == CKKSMI_NORM_LAYER ? m0 * A.inv_d : 0.0f;
            m1 *= A.inv_d;
        }
        if (mine) {
            back_store<T, LAYER, ELEMENT>(A, w, at, row, B, now.st, m0, m1);
            back_columns<LAYER, ELEMENT>(A, B, columns);
        }
    }
    if (!A.sums) return;
    if constexpr (GROUPS > 1) {  // the workgroup's groups, added in their order
        __shared__ float others[256][8];
#pragma unroll
        for (int k = 0; k < NORM_SUMS; k++) {
            if (!(A.sums >> k & 1)) continue;
#pragma unroll
            for (int e = 0; e < 8; e++) others[threadIdx.x][e] = columns[k][e];
            __syncthreads();
            if (threadIdx.x < LANES)
                for (int g = 1; g < GROUPS; g++)
#pragma unroll
                    for (int e = 0; e < 8; e++) columns[k][e] += others[g * LANES + threadIdx.x][e];
            __syncthreads();
        }
        if (threadIdx.x >= LANES) return;
    }
    put_columns(A, blockIdx.x, at, columns);
}

// ---- rows longer than the registers of a workgroup hold
#define NORM_LONG 512  // threads a row
template <class T> __global__ void __launch_bounds__(NORM_LONG) norm_forward_long_kernel(NormArgs A) {
    __shared__ float slots[2][NORM_LONG / 64][2];
    RowSums<NORM_LONG> sums(slots);
    const int octs = (A.d + 7) / 8;
    for (int row = blockIdx.x; row < A.M; row += gridDim.x) {
        const T *x = (const T *)(A.x + (size_t)row * A.ld_x), *f = (const T *)(A.f + (size_t)row * A.ld_f);
        // mean and s of what value(oct, v) gives (zeros beyond the row)
        auto stats = [&](int kind, auto value, float &mean, float &s) {
            mean = 0.0f;
            float v[8], q = 0.0f, left = 0.0f;
            if (kind == CKKSMI_NORM_LAYER) {
                for (int o = threadIdx.x; o < octs; o += NORM_LONG) {
                    value(8 * o, v);
#pragma unroll
                    for (int e = 0; e < 8; e++) mean += v[e];
                }
                sums(mean);
                mean *= A.inv_d;
            }
            for (int o = threadIdx.x; o < octs; o += NORM_LONG) {
                value(8 * o, v);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float c = 8 * o + e < A.d ? v[e] - mean : 0.0f;
                    q = fmaf(c, c, q);
                    left += c;
                }
            }
            sums(q, left);
            if (kind == CKKSMI_NORM_LAYER) right_mean(A, left, mean, q);
            s = 1.0f / sqrtf(q * A.inv_d + A.eps);
        };
        auto load = [&](const T *p, int at, float (&v)[8]) {
            Oct<T> o;
            get8(p + at, A.d - at, o);
            floats(o, v);
        };
        float mean1 = 0.0f, s1 = 1.0f, mean2 = 0.0f, s2 = 1.0f;
        if (A.post != CKKSMI_NORM_NONE) stats(A.post, [&](int at, float (&v)[8]) { load(f, at, v); }, mean1, s1);
        auto sum = [&](int at, float (&v)[8]) {  // r
            if (!A.f) return load(x, at, v);
            float xs[8], g[8], h, y;
            NormWeights w;
            norm_weights<T, true>(A, at, w);
            load(f, at, v);
            load(x, at, xs);
            if (A.gate_kind == CKKSMI_GATE_ELEMENT) load((const T *)(A.gate + (size_t)row * A.ld_gate), at, g);
            else
#pragma unroll
                for (int e = 0; e < 8; e++) g[e] = w.g[e];
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = at + e < A.d ? norm_sum<true>(A, w, e, xs[e], v[e], g[e], mean1, s1, h, y) : 0.0f;
        };
        if (A.pre != CKKSMI_NORM_NONE) stats(A.pre, sum, mean2, s2);
        // (r may be x: a thread reads its elements for the last time before it writes them)
        for (int o = threadIdx.x; o < octs; o += NORM_LONG) {
            const int at = 8 * o;
            float v[8], w[8], b[8];
            sum(at, v);
            if (A.r) put8((T *)(A.r + (size_t)row * A.ld_r) + at, A.d - at, v);
            if (A.pre == CKKSMI_NORM_NONE) continue;
            weights8<T>(A.pre_w, A.w_f32, at, A.d - at, 1.0f, w);
            weights8<T>(A.pre_b, A.w_f32, at, A.d - at, 0.0f, b);
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = fmaf((v[e] - mean2) * s2, w[e], b[e]);
            put8((T *)(A.n + (size_t)row * A.ld_n) + at, A.d - at, v);
        }
        if (A.stats && threadIdx.x == 0) *(f32x4 *)(A.stats + 4 * (size_t)row) = f32x4{mean1, s1, mean2, s2};
    }
}

// 8 elements of a row on their way back, from memory, and their columns' weights
template <class T, bool ELEMENT> __device__ __forceinline__ void back_load(const NormArgs &A, int at, size_t row, const f32x4 &st, NormWeights &w, NormBack &B) {
    const int left = A.d - at;
    Oct<T> x, f{}, g{}, dr{}, dn{};
    get8((const T *)(A.x + row * A.ld_x) + at, left, x);
    if (A.f) get8((const T *)(A.f + row * A.ld_f) + at, left, f);
    if (ELEMENT) get8((const T *)(A.gate + row * A.ld_gate) + at, left, g);
    if (A.dr) get8((const T *)(A.dr + row * A.ld_dr) + at, left, dr);
    if (A.dn) get8((const T *)(A.dn + row * A.ld_dn) + at, left, dn);
    norm_weights<T, true>(A, at, w);
    back_begin<T, true, ELEMENT>(A, w, x, f, g, dr, dn, st, B);
}
template <class T, bool ELEMENT> __global__ void __launch_bounds__(NORM_LONG) norm_backward_long_kernel(NormArgs A) {
    __shared__ float slots[2][NORM_LONG / 64][2];
    RowSums<NORM_LONG> sums(slots);
    const int octs = (A.d + 7) / 8;
    for (int row = blockIdx.x; row < A.M; row += gridDim.x) {
        const f32x4 st = *(const f32x4 *)(A.stats + 4 * (size_t)row);
        f32x4 m = {0, 0, 0, 0};
        NormBack B;
        NormWeights w;
        if (A.pre != CKKSMI_NORM_NONE) {
            float a = 0.0f, b = 0.0f;
            for (int o = threadIdx.x; o < octs; o += NORM_LONG) {
                back_load<T, ELEMENT>(A, 8 * o, row, st, w, B);
                back_pre_sums<true>(A, w, B, A.d - 8 * o, a, b);
            }
            sums(a, b);
            m[0] = A.pre == CKKSMI_NORM_LAYER ? a * A.inv_d : 0.0f;
            m[1] = b * A.inv_d;
        }
        if (A.post != CKKSMI_NORM_NONE) {
            float a = 0.0f, b = 0.0f;
            for (int o = threadIdx.x; o < octs; o += NORM_LONG) {
                back_load<T, ELEMENT>(A, 8 * o, row, st, w, B);
                back_r<true>(A, w, B, st, m[0], m[1]);
                back_post_sums<true, ELEMENT>(A, w, B, A.d - 8 * o, a, b);
            }
            sums(a, b);
            m[2] = A.post == CKKSMI_NORM_LAYER ? a * A.inv_d : 0.0f;
            m[3] = b * A.inv_d;
        }
        for (int o = threadIdx.x; o < octs; o += NORM_LONG) {
            back_load<T, ELEMENT>(A, 8 * o, row, st, w, B);
            back_r<true>(A, w, B, st, m[0], m[1]);
            back_store<T, true, ELEMENT>(A, w, 8 * o, row, B, st, m[2], m[3]);
        }
        if (A.coef && threadIdx.x == 0) *(f32x4 *)(A.coef + 4 * (size_t)row) = m;
    }
}
// column sums of rows that the kernel above has taken: a wave holds 512 columns, the workgroups' waves (blockIdx.y) share the rows
template <class T, bool ELEMENT> __global__ void __launch_bounds__(256) norm_columns_kernel(NormArgs A) {
    const int at = 8 * (blockIdx.x * 64 + (threadIdx.x & 63)), wave = blockIdx.y * 4 + (threadIdx.x >> 6);
    if (at >= A.d) return;
    float columns[NORM_SUMS][8];
#pragma unroll
    for (int k = 0; k < NORM_SUMS; k++)
#pragma unroll
        for (int e = 0; e < 8; e++) columns[k][e] = 0.0f;
    for (int row = wave; row < A.M; row += gridDim.y * 4) {
        const f32x4 st = *(const f32x4 *)(A.stats + 4 * (size_t)row), m = *(const f32x4 *)(A.coef + 4 * (size_t)row);
        NormBack B;
        NormWeights w;
        back_load<T, ELEMENT>(A, at, row, st, w, B);
        back_r<true>(A, w, B, st, m[0], m[1]);
        back_columns<true, ELEMENT>(A, B, columns);
    }
    put_columns(A, wave, at, columns);
}

// The groups' column sums added in their order, 16 waves sharing the groups (their sums are added in the waves' order), and the gradients that come from
// them: 64 columns a workgroup
struct NormJoinArgs {
    const float *part;
    size_t ld_part;
    int groups, vectors, d, w_f32, accumulate;
    struct Out {
        char *o;
        int first, second;           // which sums; second: -1 if there is one only
        const char *by, *second_by;  // columns' factors (null: 1)
    } out[NORM_SUMS + 1];
};
template <class T> __global__ void __launch_bounds__(1024) norm_join_kernel(NormJoinArgs A) {
    __shared__ float sums[2][16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    const NormJoinArgs::Out &O = A.out[blockIdx.y];
    float s[2] = {0.0f, 0.0f};
    if (c < A.d)
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int k = i ? O.second : O.first;
            if (k < 0) continue;
            const float *p = A.part + (size_t)k * A.ld_part + c;
            const size_t next = (size_t)A.vectors * A.ld_part;
#pragma unroll 8
            for (int g = wave; g < A.groups; g += 16) s[i] += p[g * next];
        }
    sums[0][wave][lane] = s[0];
    sums[1][wave][lane] = s[1];
    __syncthreads();
    if (wave || c >= A.d) return;
#pragma unroll
    for (int w = 1; w < 16; w++) {
        s[0] += sums[0][w][lane];
        s[1] += sums[1][w][lane];
    }
    auto factor = [&](const char *w) { return !w ? 1.0f : A.w_f32 || sizeof(T) == 4 ? ((const float *)w)[c] : (float)((const T *)w)[c]; };
    float v = s[0] * factor(O.by);
    if (O.second >= 0) v += s[1] * factor(O.second_by);
    if (A.w_f32 || sizeof(T) == 4) {
        float *o = (float *)O.o + c;
        *o = A.accumulate ? *o + v : v;
    } else {
        T *o = (T *)O.o + c;
        *o = (T)(A.accumulate ? (float)*o + v : v);
    }
}
