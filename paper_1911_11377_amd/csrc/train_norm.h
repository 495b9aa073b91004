// Norms before and after a block with its gate and residual sum: r = a x + b gate N1(f), n = N2(r), and their backward pass.
//
// A row's norm needs all of the row before its first result: a group of threads holds a row in registers (8 neighbouring elements at a
// time a thread, V times), so every operand is read once.  With h = (v - mean) s, s = 1 / sqrt(mean (v - mean)^2 + eps), the gradient of
// N(v) = h w + b by v is, for g = dy w,
//     dv = (g - mean(g) - h mean(g h)) s          (rms: without the first mean)
// The forward pass saves each row's two means and two s; the backward pass forms h of both norms again from x and f and needs two rounds of sums
// over the row.  Gradients of weights, biases and a channel gate are sums over rows: a thread keeps its columns' sums over all rows that
// its group takes, groups' sums go to memory once, and a second kernel adds them in their order.
// Longer rows than registers hold are read once for each sum; their column sums take a pass of their own.
// Bound by memory.
#pragma once
#include "train_types.h"

struct NormArgs {
    const char *x, *f, *gate;
    const char *post_w, *post_b, *pre_w, *pre_b;
    char *r, *n;
    float *stats;  // [rows][4]: mean and s of f, of r
    const char *dr, *dn;
    char *dx, *df, *dgate;
    float *part;   // [groups][vectors][ld_part]
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
enum NormSum { SUM_POST_W = 1, SUM_POST_B = 2, SUM_PRE_W = 4, SUM_PRE_B = 8, SUM_GATE = 16, NORM_SUMS = 5 };

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

// mean and s of a row's values that the group holds (elements beyond the row are zeros)
template <int LANES, int V> __device__ __forceinline__ void row_stats(const NormArgs &A, int kind, int t, const float (&v)[V][8], RowSums<LANES> &sums, float &mean, float &s) {
    mean = 0.0f;
    if (kind == CKKSMI_NORM_LAYER) {
#pragma unroll
        for (int j = 0; j < V; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) mean += v[j][e];
        sums(mean);
        mean *= A.inv_d;
    }
    float q = 0.0f;
#pragma unroll
    for (int j = 0; j < V; j++)
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float c = 8 * (t + LANES * j) + e < A.d ? v[j][e] - mean : 0.0f;
            q += c * c;
        }
    sums(q);
    s = 1.0f / sqrtf(q * A.inv_d + A.eps);
}

// Rows are taken by groups of LANES threads, 8 * V * LANES elements at most each; GROUPS of them in a workgroup
template <int LANES> struct NormShape {
    static constexpr int THREADS = LANES > 64 ? LANES : 256, GROUPS = THREADS / LANES;
};

template <class T, int LANES, int V>
__global__ void __launch_bounds__(NormShape<LANES>::THREADS) norm_forward_kernel(NormArgs A) {
    constexpr int GROUPS = NormShape<LANES>::GROUPS;
    __shared__ float slots[2][RowSums<LANES>::WAVES][2];
    RowSums<LANES> sums(slots);
    const int t = threadIdx.x % LANES, group = threadIdx.x / LANES;
    struct Row { Oct<T> x[V], f[V]; };
    auto load = [&](Row &w, int row) {
        const T *x = (const T *)(A.x + (size_t)row * A.ld_x), *f = (const T *)(A.f + (size_t)row * A.ld_f);
#pragma unroll
        for (int j = 0; j < V; j++) {
            const int at = 8 * (t + LANES * j);
            get8(x + at, A.d - at, w.x[j]);
            if (A.f) get8(f + at, A.d - at, w.f[j]);
        }
    };
    Row next;
    const int stride = gridDim.x * GROUPS;
    load(next, min((int)blockIdx.x * GROUPS + group, A.M - 1));
    for (int first = blockIdx.x * GROUPS; first < A.M; first += stride) {
        // (a group without a row repeats the last one and stores nothing)
        const int row = min(first + group, A.M - 1);
        const bool mine = first + group < A.M;
        const Row now = next;
        if (first < A.M - stride) load(next, min(first + stride + group, A.M - 1));
        float v[V][8];
        float mean1 = 0.0f, s1 = 1.0f, mean2 = 0.0f, s2 = 1.0f;
        if (A.f) {
#pragma unroll
            for (int j = 0; j < V; j++) floats(now.f[j], v[j]);
            if (A.post != CKKSMI_NORM_NONE) row_stats<LANES, V>(A, A.post, t, v, sums, mean1, s1);
#pragma unroll
            for (int j = 0; j < V; j++) {
                const int at = 8 * (t + LANES * j);
                float x[8], w[8], b[8], g[8];
                floats(now.x[j], x);
                if (A.post != CKKSMI_NORM_NONE) {
                    weights8<T>(A.post_w, A.w_f32, at, A.d - at, 1.0f, w);
                    weights8<T>(A.post_b, A.w_f32, at, A.d - at, 0.0f, b);
#pragma unroll
                    for (int e = 0; e < 8; e++) v[j][e] = (v[j][e] - mean1) * s1 * w[e] + b[e];
                }
                if (A.gate_kind == CKKSMI_GATE_CHANNEL) weights8<T>(A.gate, A.w_f32, at, A.d - at, 1.0f, g);
                else if (A.gate_kind == CKKSMI_GATE_ELEMENT) {
                    Oct<T> o;
                    get8((const T *)(A.gate + (size_t)row * A.ld_gate) + at, A.d - at, o);
                    floats(o, g);
                }
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    if (A.gate_kind != CKKSMI_GATE_NONE) v[j][e] *= g[e];
                    v[j][e] = at + e < A.d ? A.a * x[e] + A.b * v[j][e] : 0.0f;
                }
                if (A.r && mine) put8((T *)(A.r + (size_t)row * A.ld_r) + at, A.d - at, v[j]);
            }
        } else
#pragma unroll
            for (int j = 0; j < V; j++) floats(now.x[j], v[j]);
        if (A.pre != CKKSMI_NORM_NONE) {
            row_stats<LANES, V>(A, A.pre, t, v, sums, mean2, s2);
#pragma unroll
            for (int j = 0; j < V; j++) {
                const int at = 8 * (t + LANES * j);
                float w[8], b[8];
                weights8<T>(A.pre_w, A.w_f32, at, A.d - at, 1.0f, w);
                weights8<T>(A.pre_b, A.w_f32, at, A.d - at, 0.0f, b);
#pragma unroll
                for (int e = 0; e < 8; e++) v[j][e] = (v[j][e] - mean2) * s2 * w[e] + b[e];
                if (mine) put8((T *)(A.n + (size_t)row * A.ld_n) + at, A.d - at, v[j]);
            }
        }
        if (A.stats && mine && t == 0) *(f32x4 *)(A.stats + 4 * (size_t)row) = f32x4{mean1, s1, mean2, s2};
    }
}

// One row's 8 elements on their way back
struct NormBack {
    float h1[8], y[8], g[8], h2[8], dt[8], dn[8];
};
// h of both norms, N1(f) and the gate; dr in dt
template <class T>
__device__ __forceinline__ void back_begin(const NormArgs &A, int at, const Oct<T> &ox, const Oct<T> &of, const Oct<T> &og, const Oct<T> &odr, const Oct<T> &odn, const f32x4 &st,
                                           NormBack &B) {
    const int left = A.d - at;
    float x[8];
    floats(ox, x);
    floats(odr, B.dt);
    floats(odn, B.dn);
    if (A.f) {
        floats(of, B.y);
        if (A.post != CKKSMI_NORM_NONE) {
            float w[8], b[8];
            weights8<T>(A.post_w, A.w_f32, at, left, 1.0f, w);
            weights8<T>(A.post_b, A.w_f32, at, left, 0.0f, b);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                B.h1[e] = (B.y[e] - st[0]) * st[1];
                B.y[e] = B.h1[e] * w[e] + b[e];
            }
        }
        if (A.gate_kind == CKKSMI_GATE_CHANNEL) weights8<T>(A.gate, A.w_f32, at, left, 1.0f, B.g);
        else if (A.gate_kind == CKKSMI_GATE_ELEMENT) floats(og, B.g);
    }
    if (A.pre != CKKSMI_NORM_NONE)
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float y = A.gate_kind != CKKSMI_GATE_NONE ? B.y[e] * B.g[e] : B.y[e];
            const float r = A.f ? A.a * x[e] + A.b * y : x[e];
            B.h2[e] = (r - st[2]) * st[3];
        }
}
// what the norm of n sends back: its share of mean(g), mean(g h)
template <class T> __device__ __forceinline__ void back_pre_sums(const NormArgs &A, int at, const NormBack &B, float &s0, float &s1) {
    float w[8];
    weights8<T>(A.pre_w, A.w_f32, at, A.d - at, 1.0f, w);
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const float g = at + e < A.d ? B.dn[e] * w[e] : 0.0f;
        s0 += g;
        s1 += at + e < A.d ? g * B.h2[e] : 0.0f;
    }
}
// dt: the gradient of r
template <class T> __device__ __forceinline__ void back_r(const NormArgs &A, int at, NormBack &B, const f32x4 &st, float m0, float m1) {
    if (A.pre == CKKSMI_NORM_NONE) return;
    float w[8];
    weights8<T>(A.pre_w, A.w_f32, at, A.d - at, 1.0f, w);
#pragma unroll
    for (int e = 0; e < 8; e++) B.dt[e] += (B.dn[e] * w[e] - m0 - B.h2[e] * m1) * st[3];
}
// gradient of N1(f)
__device__ __forceinline__ float back_y(const NormArgs &A, const NormBack &B, int e) {
    const float du = B.dt[e] * A.b;
    return A.gate_kind != CKKSMI_GATE_NONE ? du * B.g[e] : du;
}
template <class T> __device__ __forceinline__ void back_post_sums(const NormArgs &A, int at, const NormBack &B, float &s0, float &s1) {
    float w[8];
    weights8<T>(A.post_w, A.w_f32, at, A.d - at, 1.0f, w);
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const float g = at + e < A.d ? back_y(A, B, e) * w[e] : 0.0f;
        s0 += g;
        s1 += at + e < A.d ? g * B.h1[e] : 0.0f;
    }
}
// gradients of the elements to memory
template <class T> __device__ __forceinline__ void back_store(const NormArgs &A, int at, size_t row, const NormBack &B, const f32x4 &st, float m0, float m1) {
    const int left = A.d - at;
    float o[8];
    if (A.dx) {
#pragma unroll
        for (int e = 0; e < 8; e++) o[e] = A.f ? B.dt[e] * A.a : B.dt[e];
        put8((T *)(A.dx + row * A.ld_dx) + at, left, o);
    }
    if (!A.f) return;
    if (A.dgate) {
#pragma unroll
        for (int e = 0; e < 8; e++) o[e] = B.dt[e] * A.b * B.y[e];
        put8((T *)(A.dgate + row * A.ld_dgate) + at, left, o);
    }
    if (A.df) {
        if (A.post != CKKSMI_NORM_NONE) {
            float w[8];
            weights8<T>(A.post_w, A.w_f32, at, left, 1.0f, w);
#pragma unroll
            for (int e = 0; e < 8; e++) o[e] = (back_y(A, B, e) * w[e] - m0 - B.h1[e] * m1) * st[1];
        } else
#pragma unroll
            for (int e = 0; e < 8; e++) o[e] = back_y(A, B, e);
        put8((T *)(A.df + row * A.ld_df) + at, left, o);
    }
}
// a row's terms of the column sums
__device__ __forceinline__ void back_columns(const NormArgs &A, const NormBack &B, float (&sum)[NORM_SUMS][8]) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
        if (A.sums & SUM_POST_W) sum[0][e] += back_y(A, B, e) * B.h1[e];
        if (A.sums & SUM_POST_B) sum[1][e] += back_y(A, B, e);
        if (A.sums & SUM_PRE_W) sum[2][e] += B.dn[e] * B.h2[e];
        if (A.sums & SUM_PRE_B) sum[3][e] += B.dn[e];
        if (A.sums & SUM_GATE) sum[4][e] += B.dt[e] * A.b * B.y[e];
    }
}
// a group's column sums to memory
__device__ __forceinline__ void put_columns(const NormArgs &A, size_t group, int at, const float (&sum)[NORM_SUMS][8]) {
    float *p = A.part + group * A.vectors * A.ld_part + at;
#pragma unroll
    for (int k = 0; k < NORM_SUMS; k++)
        if (A.sums >> k & 1) {
            if (at < A.d) store_oct(p, sum[k]);
            p += A.ld_part;
        }
}

template <class T, int LANES, int V>
__global__ void __launch_bounds__(NormShape<LANES>::THREADS) norm_backward_kernel(NormArgs A) {
    constexpr int GROUPS = NormShape<LANES>::GROUPS;
    __shared__ float slots[2][RowSums<LANES>::WAVES][2];
    RowSums<LANES> sums(slots);
    const int t = threadIdx.x % LANES, group = threadIdx.x / LANES;
    struct Row { Oct<T> x[V], f[V], g[V], dr[V], dn[V]; f32x4 st; };
    auto load = [&](Row &w, int row_) {
        const size_t row = row_;
        w.st = *(const f32x4 *)(A.stats + 4 * row);
#pragma unroll
        for (int j = 0; j < V; j++) {
            const int at = 8 * (t + LANES * j), left = A.d - at;
            w.dr[j] = w.dn[j] = Oct<T>{};
            get8((const T *)(A.x + row * A.ld_x) + at, left, w.x[j]);
            if (A.f) get8((const T *)(A.f + row * A.ld_f) + at, left, w.f[j]);
            if (A.gate_kind == CKKSMI_GATE_ELEMENT) get8((const T *)(A.gate + row * A.ld_gate) + at, left, w.g[j]);
            if (A.dr) get8((const T *)(A.dr + row * A.ld_dr) + at, left, w.dr[j]);
            if (A.dn) get8((const T *)(A.dn + row * A.ld_dn) + at, left, w.dn[j]);
        }
    };
    float columns[V][NORM_SUMS][8];
#pragma unroll
    for (int j = 0; j < V; j++)
#pragma unroll
        for (int k = 0; k < NORM_SUMS; k++)
#pragma unroll
            for (int e = 0; e < 8; e++) columns[j][k][e] = 0.0f;
    Row next;
    const int stride = gridDim.x * GROUPS;
    load(next, min((int)blockIdx.x * GROUPS + group, A.M - 1));
    for (int first = blockIdx.x * GROUPS; first < A.M; first += stride) {
        const int row = min(first + group, A.M - 1);
        const bool mine = first + group < A.M;
        const Row now = next;
        if (first < A.M - stride) load(next, min(first + stride + group, A.M - 1));
        NormBack B[V];
#pragma unroll
        for (int j = 0; j < V; j++) back_begin<T>(A, 8 * (t + LANES * j), now.x[j], now.f[j], now.g[j], now.dr[j], now.dn[j], now.st, B[j]);
        float m0 = 0.0f, m1 = 0.0f;
        if (A.pre != CKKSMI_NORM_NONE) {
#pragma unroll
            for (int j = 0; j < V; j++) back_pre_sums<T>(A, 8 * (t + LANES * j), B[j], m0, m1);
            sums(m0, m1);
            m0 = A.pre == CKKSMI_NORM_LAYER ? m0 * A.inv_d : 0.0f;
            m1 *= A.inv_d;
#pragma unroll
            for (int j = 0; j < V; j++) back_r<T>(A, 8 * (t + LANES * j), B[j], now.st, m0, m1);
        }
        m0 = m1 = 0.0f;
        if (A.f && A.post != CKKSMI_NORM_NONE) {
#pragma unroll
            for (int j = 0; j < V; j++) back_post_sums<T>(A, 8 * (t + LANES * j), B[j], m0, m1);
            sums(m0, m1);
            m0 = A.post == CKKSMI_NORM_LAYER ? m0 * A.inv_d : 0.0f;
            m1 *= A.inv_d;
        }
        if (mine)
#pragma unroll
            for (int j = 0; j < V; j++) {
                back_store<T>(A, 8 * (t + LANES * j), row, B[j], now.st, m0, m1);
                back_columns(A, B[j], columns[j]);
            }
    }
    if (A.sums)
#pragma unroll
        for (int j = 0; j < V; j++) put_columns(A, (size_t)blockIdx.x * GROUPS + group, 8 * (t + LANES * j), columns[j]);
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
            float v[8], q = 0.0f;
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
                    q += c * c;
                }
            }
            sums(q);
            s = 1.0f / sqrtf(q * A.inv_d + A.eps);
        };
        auto load = [&](const T *p, int at, float (&v)[8]) {
            Oct<T> o;
            get8(p + at, A.d - at, o);
            floats(o, v);
        };
        float mean1 = 0.0f, s1 = 1.0f, mean2 = 0.0f, s2 = 1.0f;
        if (A.f && A.post != CKKSMI_NORM_NONE) stats(A.post, [&](int at, float (&v)[8]) { load(f, at, v); }, mean1, s1);
        auto sum = [&](int at, float (&v)[8]) {  // r
            if (!A.f) return load(x, at, v);
            float xs[8], w[8], b[8], g[8];
            load(f, at, v);
            load(x, at, xs);
            if (A.post != CKKSMI_NORM_NONE) {
                weights8<T>(A.post_w, A.w_f32, at, A.d - at, 1.0f, w);
                weights8<T>(A.post_b, A.w_f32, at, A.d - at, 0.0f, b);
#pragma unroll
                for (int e = 0; e < 8; e++) v[e] = (v[e] - mean1) * s1 * w[e] + b[e];
            }
            if (A.gate_kind == CKKSMI_GATE_CHANNEL) weights8<T>(A.gate, A.w_f32, at, A.d - at, 1.0f, g);
            else if (A.gate_kind == CKKSMI_GATE_ELEMENT) load((const T *)(A.gate + (size_t)row * A.ld_gate), at, g);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                if (A.gate_kind != CKKSMI_GATE_NONE) v[e] *= g[e];
                v[e] = at + e < A.d ? A.a * xs[e] + A.b * v[e] : 0.0f;
            }
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
            for (int e = 0; e < 8; e++) v[e] = (v[e] - mean2) * s2 * w[e] + b[e];
            put8((T *)(A.n + (size_t)row * A.ld_n) + at, A.d - at, v);
        }
        if (A.stats && threadIdx.x == 0) *(f32x4 *)(A.stats + 4 * (size_t)row) = f32x4{mean1, s1, mean2, s2};
    }
}

// 8 elements of a row on their way back, from memory
template <class T> __device__ __forceinline__ void back_load(const NormArgs &A, int at, size_t row, const f32x4 &st, NormBack &B) {
    const int left = A.d - at;
    Oct<T> x, f{}, g{}, dr{}, dn{};
    get8((const T *)(A.x + row * A.ld_x) + at, left, x);
    if (A.f) get8((const T *)(A.f + row * A.ld_f) + at, left, f);
    if (A.gate_kind == CKKSMI_GATE_ELEMENT) get8((const T *)(A.gate + row * A.ld_gate) + at, left, g);
    if (A.dr) get8((const T *)(A.dr + row * A.ld_dr) + at, left, dr);
    if (A.dn) get8((const T *)(A.dn + row * A.ld_dn) + at, left, dn);
    back_begin<T>(A, at, x, f, g, dr, dn, st, B);
}
template <class T> __global__ void __launch_bounds__(NORM_LONG) norm_backward_long_kernel(NormArgs A) {
    __shared__ float slots[2][NORM_LONG / 64][2];
    RowSums<NORM_LONG> sums(slots);
    const int octs = (A.d + 7) / 8;
    for (int row = blockIdx.x; row < A.M; row += gridDim.x) {
        const f32x4 st = *(const f32x4 *)(A.stats + 4 * (size_t)row);
        f32x4 m = {0, 0, 0, 0};
        NormBack B;
        if (A.pre != CKKSMI_NORM_NONE) {
            float a = 0.0f, b = 0.0f;
            for (int o = threadIdx.x; o < octs; o += NORM_LONG) {
                back_load<T>(A, 8 * o, row, st, B);
                back_pre_sums<T>(A, 8 * o, B, a, b);
            }
            sums(a, b);
            m[0] = A.pre == CKKSMI_NORM_LAYER ? a * A.inv_d : 0.0f;
            m[1] = b * A.inv_d;
        }
        if (A.f && A.post != CKKSMI_NORM_NONE) {
            float a = 0.0f, b = 0.0f;
            for (int o = threadIdx.x; o < octs; o += NORM_LONG) {
                back_load<T>(A, 8 * o, row, st, B);
                back_r<T>(A, 8 * o, B, st, m[0], m[1]);
                back_post_sums<T>(A, 8 * o, B, a, b);
            }
            sums(a, b);
            m[2] = A.post == CKKSMI_NORM_LAYER ? a * A.inv_d : 0.0f;
            m[3] = b * A.inv_d;
        }
        for (int o = threadIdx.x; o < octs; o += NORM_LONG) {
            back_load<T>(A, 8 * o, row, st, B);
            back_r<T>(A, 8 * o, B, st, m[0], m[1]);
            back_store<T>(A, 8 * o, row, B, st, m[2], m[3]);
        }
        if (A.coef && threadIdx.x == 0) *(f32x4 *)(A.coef + 4 * (size_t)row) = m;
    }
}
// column sums of rows that the kernel above has taken: a wave holds 512 columns, the workgroups' waves (blockIdx.y) share the rows
template <class T> __global__ void __launch_bounds__(256) norm_columns_kernel(NormArgs A) {
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
        back_load<T>(A, at, row, st, B);
        back_r<T>(A, at, B, st, m[0], m[1]);
        back_columns(A, B, columns);
    }
    put_columns(A, wave, at, columns);
}

// The groups' column sums added in their order: 64 columns a workgroup, 16 waves share the groups, and their sums are added in the waves' order
struct NormJoinArgs {
    const float *part;
    size_t ld_part;
    int groups, vectors, d, f32_out, accumulate;
    char *out[NORM_SUMS];  // of the vectors that are there
};
template <class T> __global__ void __launch_bounds__(1024) norm_join_kernel(NormJoinArgs A) {
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane, k = blockIdx.y;
    float s = 0.0f;
    if (c < A.d) {
        const float *p = A.part + (size_t)k * A.ld_part + c;
        const size_t next = (size_t)A.vectors * A.ld_part;
#pragma unroll 8
        for (int g = wave; g < A.groups; g += 16) s += p[g * next];
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave || c >= A.d) return;
#pragma unroll
    for (int w = 1; w < 16; w++) s += sums[w][lane];
    if (A.f32_out || sizeof(T) == 4) {
        float *o = (float *)A.out[k] + c;
        *o = A.accumulate ? *o + s : s;
    } else {
        T *o = (T *)A.out[k] + c;
        *o = (T)(A.accumulate ? (float)*o + s : s);
    }
}
