// AdamW over many tensors in one launch.
//
// Every element is read once and written once, with some 20 operations in between (60 with 8-bit states): memory bounds
// the step.  A workgroup takes 4096 neighbouring elements of one tensor, found in a table of tensors that travels as a kernel
// argument; a wave takes 256 of them at a time, 4 neighbouring ones a lane, which is one block of the 8-bit states: its
// largest magnitudes are found among the wave's lanes and no step needs LDS or a second pass.
// Products and sums are rounded one by one (no fused multiply-add): an element's result depends on nothing but its inputs.
#pragma once
#include "train_types.h"

#define TA_TENSORS 48  // of one launch
#define TA_CHUNK 4096  // elements of a workgroup
static_assert(CKKSMI_STATE_BLOCK == 256, "a block is 64 lanes x 4 elements");

struct AdamwArgs {
    ckksmi_adamw_tensor t[TA_TENSORS];
    unsigned first[TA_TENSORS + 1];  // workgroups of the tensors before
    int n;
    int tensor0;  // index of t[0] in the call
    int copy_f16;
    unsigned key;  // of the seed
    float beta1, rest1, beta2, rest2, decay, size, root, eps, grad_scale;
    const int *skip;
};

__host__ __device__ __forceinline__ unsigned adamw_mix(unsigned h) {
    h ^= h >> 16;
    h *= 0x6A09E667u;  // fractions of the roots of 2 and 3
    h ^= h >> 15;
    h *= 0xBB67AE85u;
    return h ^ (h >> 16);
}

// 4 elements from index i of n on; beyond the end zeros
template <class T> __device__ __forceinline__ void load4(const T *p, int64_t i, int64_t n, bool vec, T (&x)[4]) {
    if (vec && i + 4 <= n) {
        struct alignas(4 * sizeof(T)) V { T v[4]; } o = *(const V *)(p + i);
#pragma unroll
        for (int e = 0; e < 4; e++) x[e] = o.v[e];
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; e++) x[e] = i + e < n ? p[i + e] : (T)0;
}
template <class T> __device__ __forceinline__ void store4(T *p, int64_t i, int64_t n, bool vec, const T (&x)[4]) {
    if (vec && i + 4 <= n) {
        struct alignas(4 * sizeof(T)) V { T v[4]; } o;
#pragma unroll
        for (int e = 0; e < 4; e++) o.v[e] = x[e];
        *(V *)(p + i) = o;
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; e++)
        if (i + e < n) p[i + e] = x[e];
}
template <class T> __device__ __forceinline__ bool at4(const T *p) { return ((uintptr_t)p & (4 * sizeof(T) - 1)) == 0; }

// largest word of a wave, in every lane
__device__ __forceinline__ unsigned wave_max(unsigned v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const unsigned w = (unsigned)__shfl_xor((int)v, d);
        v = v > w ? v : w;
    }
    return v;
}

// 8-bit codes: FRACTION bits behind the leading one, 4 bits of exponent; see ckksmi_train.h
template <int FRACTION> __device__ __forceinline__ float code_value(unsigned c) {
    constexpr unsigned one = 1u << FRACTION;
    const unsigned e = c >> FRACTION;
    return (float)(e == 0 ? c : (one + (c & (one - 1))) << (e - 1));
}
// z: magnitude in units, below 2^(16 + FRACTION); random: 16 bits.  The word of z (of z + one below `one`, where codes are evenly spaced)
// holds the code in its upper bits; random bits below them are added and cut off
template <int FRACTION> __device__ __forceinline__ unsigned code_of(float z, unsigned random) {
    constexpr unsigned one = 1u << FRACTION, shift = 23 - FRACTION, base = (127 + FRACTION) << FRACTION;
    const bool small = z < (float)one;
    const unsigned w = __float_as_uint(small ? z + (float)one : z) + (random << (shift - 16));
    const unsigned c = (w >> shift) - (small ? base : base - one);
    return c < 16 * one - 1 ? c : 16 * one - 1;
}
// unit and its inverse for a block whose largest magnitude has the word `top` (NaN and infinity have the largest words of all)
template <int FRACTION> __device__ __forceinline__ float block_unit(unsigned top, float &inverse) {
    const float unit = __uint_as_float(top) * (float)(1.0 / (double)(((2 << FRACTION) - 1) << 14));
    const bool held = unit >= 1e-36f;  // below: the block is held as zeros
    inverse = held ? 1.0f / unit : 0.0f;
    return held ? unit : 0.0f;
}

struct AdamwElement { float p, m, v; };
__device__ __forceinline__ AdamwElement adamw_element(const AdamwArgs &A, float p, float grad, float m, float v) {
    AdamwElement o;
    const float g = grad * A.grad_scale;
    o.m = m * A.beta1 + g * A.rest1;
    o.v = v * A.beta2 + g * g * A.rest2;
    o.p = p * A.decay - o.m / (sqrtf(o.v) * A.root + A.eps) * A.size;
    return o;
}

template <class P, class G, int BITS>
__global__ void __launch_bounds__(256) adamw_kernel(AdamwArgs A) {
    if (A.skip && *A.skip) return;
    int lo = 0, hi = A.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (A.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    const ckksmi_adamw_tensor &t = A.t[lo];
    const int64_t n = t.n, begin = (int64_t)(blockIdx.x - A.first[lo]) * TA_CHUNK;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    P *p = (P *)t.p;
    const G *grad = (const G *)t.grad;
    const bool p4 = at4(p), g4 = at4(grad), c4 = at4((const __bf16 *)t.copy);
    const unsigned key = adamw_mix(A.key + (unsigned)(A.tensor0 + lo));
#pragma unroll 4
    for (int b = 0; b < TA_CHUNK / 1024; b++) {
        const int64_t first = begin + (b * 4 + wave) * 256, i = first + 4 * lane;
        if (first >= n) break;
        P px[4];
        G gx[4];
        load4(p, i, n, p4, px);
        load4(grad, i, n, g4, gx);
        float q[4];
        if constexpr (BITS == 32) {
            float *m = (float *)t.m, *v = (float *)t.v;
            const bool m4 = at4(m), v4 = at4(v);
            float mx[4], vx[4];
            load4(m, i, n, m4, mx);
            load4(v, i, n, v4, vx);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const AdamwElement o = adamw_element(A, (float)px[e], (float)gx[e], mx[e], vx[e]);
                q[e] = o.p;
                mx[e] = o.m;
                vx[e] = o.v;
            }
            store4(m, i, n, m4, mx);
            store4(v, i, n, v4, vx);
        } else {
            unsigned char *m = (unsigned char *)t.m, *v = (unsigned char *)t.v;
            const bool m4 = at4(m), v4 = at4(v);
            const int64_t block = first / 256;
            unsigned char mc[4], vc[4];
            load4(m, i, n, m4, mc);
            load4(v, i, n, v4, vc);
            const float mu = t.m_unit[block], vu = t.v_unit[block];
            float mx[4], vx[4];
            unsigned mtop = 0, vtop = 0;  // words of the largest magnitudes
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float m0 = code_value<3>(mc[e] & 127u) * mu;
                const AdamwElement o = adamw_element(A, (float)px[e], (float)gx[e], mc[e] & 128u ? -m0 : m0, code_value<4>(vc[e]) * vu);
                q[e] = o.p;
                const bool in = i + e < n;
                mx[e] = in ? o.m : 0.0f;
                vx[e] = in ? o.v : 0.0f;
                const unsigned mw = __float_as_uint(mx[e]) & 0x7fffffffu, vw = __float_as_uint(vx[e]) & 0x7fffffffu;
                mtop = mtop > mw ? mtop : mw;
                vtop = vtop > vw ? vtop : vw;
            }
            mtop = wave_max(mtop);
            vtop = wave_max(vtop);
            float minv, vinv;
            const float mnew = block_unit<3>(mtop, minv), vnew = block_unit<4>(vtop, vinv);
            const bool mbad = mtop >= 0x7f800000u, vbad = vtop >= 0x7f800000u;
            const unsigned bkey = adamw_mix(adamw_mix(key + (unsigned)block) + (unsigned)(block >> 32));
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const unsigned h = adamw_mix(bkey + (4 * lane + e) * 0x9E3779B9u);
                unsigned c = code_of<3>(fabsf(mx[e]) * minv, h >> 16);
                mc[e] = (unsigned char)(mbad ? 0u : c | (mx[e] < 0.0f ? 128u : 0u));
                const float z = vx[e] * vinv;
                c = code_of<4>(z, h & 0xffffu);
                c = z > 0.0f && c == 0 ? 1u : c;
                vc[e] = (unsigned char)(vbad ? 0u : c);
            }
            store4(m, i, n, m4, mc);
            store4(v, i, n, v4, vc);
            if (lane == 0) {
                t.m_unit[block] = mbad ? __uint_as_float(0x7fc00000u) : mnew;
                t.v_unit[block] = vbad ? __uint_as_float(0x7fc00000u) : vnew;
            }
        }
#pragma unroll
        for (int e = 0; e < 4; e++) px[e] = (P)q[e];
        store4(p, i, n, p4, px);
        if (t.copy) {
            if (A.copy_f16) {
                _Float16 c[4];
#pragma unroll
                for (int e = 0; e < 4; e++) c[e] = (_Float16)q[e];
                store4((_Float16 *)t.copy, i, n, c4, c);
            } else {
                __bf16 c[4];
#pragma unroll
                for (int e = 0; e < 4; e++) c[e] = (__bf16)q[e];
                store4((__bf16 *)t.copy, i, n, c4, c);
            }
        }
    }
}

struct ReadStatesArgs {
    struct One { const unsigned char *m, *v; const float *m_unit, *v_unit; float *m_out, *v_out; int64_t n; } t[TA_TENSORS];
    unsigned first[TA_TENSORS + 1];
    int n;
};
__global__ void __launch_bounds__(256) adamw_read_kernel(ReadStatesArgs A) {
    int lo = 0, hi = A.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (A.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    const ReadStatesArgs::One &t = A.t[lo];
    const int64_t begin = (int64_t)(blockIdx.x - A.first[lo]) * TA_CHUNK;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll 4
    for (int b = 0; b < TA_CHUNK / 1024; b++) {
        const int64_t first = begin + (b * 4 + wave) * 256, i = first + 4 * lane;
        if (first >= t.n) break;
        unsigned char c[4];
        float x[4];
        if (t.m_out) {
            const float unit = t.m_unit[first / 256];
            load4(t.m, i, t.n, at4(t.m), c);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float v = code_value<3>(c[e] & 127u) * unit;
                x[e] = c[e] & 128u ? -v : v;
            }
            store4(t.m_out, i, t.n, at4(t.m_out), x);
        }
        if (t.v_out) {
            const float unit = t.v_unit[first / 256];
            load4(t.v, i, t.n, at4(t.v), c);
#pragma unroll
            for (int e = 0; e < 4; e++) x[e] = code_value<4>(c[e]) * unit;
            store4(t.v_out, i, t.n, at4(t.v_out), x);
        }
    }
}
