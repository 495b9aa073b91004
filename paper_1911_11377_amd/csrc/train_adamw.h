// AdamW over many tensors in one launch.
//
// Every element is read once and written once, with some 40 operations in between (exact quotient and root among them; 100 with
// 8-bit states).  A workgroup takes 4096 neighbouring elements of one tensor, found in a table of tensors that travels as a
// kernel argument; a wave takes 256 of them at a time, 4 neighbouring ones a lane, which is one block of the 8-bit states: its
// largest magnitudes are found among the wave's lanes and no step needs LDS or a second pass.  The next block is on its way
// while one is computed; blocks that are whole and aligned take a path without conditions (with conditions 736 us instead of
// 640 for the second case below).
// Products and sums are rounded one by one (no fused multiply-add): an element's result depends on nothing but its inputs.
// Measured: 32-bit states, 306M f32 parameters, bf16 gradients and copies 1.62 ms (28 bytes an element, 5.3 TB/s: what a copy
// reaches); 8-bit states, 221M bf16 parameters 0.64 ms (10 bytes, 3.5 TB/s: bound by its instructions), read back 0.37 ms
// (10 bytes, 6.0 TB/s, mostly writes); 160 tensors of 1 to 4M elements, 8-bit states 0.25 ms with reading back (four launches each).
#pragma once
#include <type_traits>

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

// 8-bit codes: FRACTION bits behind the leading one, 4 bits of exponent, values in units; see ckksmi_train.h.  The code is the upper
// part of the word of a 32-bit number scaled by 2^-(126 + FRACTION): codes without an exponent are its subnormal numbers
template <int FRACTION> __device__ __forceinline__ float code_value(unsigned c) {
    return __uint_as_float(c << (23 - FRACTION)) * 0x1p+100f * (float)(1u << (26 + FRACTION));
}
// z: magnitude in units; random: 16 bits, added right below the code and cut off
template <int FRACTION> __device__ __forceinline__ unsigned code_of(float z, unsigned random) {
    constexpr unsigned shift = 23 - FRACTION, most = (16u << FRACTION) - 1;
    const unsigned c = (__float_as_uint(z * 0x1p-100f * (1.0f / (float)(1u << (26 + FRACTION)))) + (random << (shift - 16))) >> shift;
    return c < most ? c : most;
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

// what a lane reads of a block
template <class P, class G, int BITS> struct AdamwLoaded;
template <class P, class G> struct AdamwLoaded<P, G, 32> { P p[4]; G g[4]; float m[4], v[4]; };
template <class P, class G> struct AdamwLoaded<P, G, 8> { P p[4]; G g[4]; unsigned char m[4], v[4]; float mu, vu; };

// a wave's share of a chunk: BLOCKS blocks from `begin` on, 1024 elements apart
template <class P, class G, int BITS, bool WHOLE, int BLOCKS>
__device__ __forceinline__ void adamw_chunk(const AdamwArgs &A, const ckksmi_adamw_tensor &t, int64_t begin, unsigned tensor) {
    typedef typename std::conditional<BITS == 8, unsigned char, float>::type State;
    const int64_t n = t.n;
    const int lane = threadIdx.x & 63;
    P *p = (P *)t.p;
    const G *grad = (const G *)t.grad;
    State *m = (State *)t.m, *v = (State *)t.v;
    const bool p4 = at4(p), g4 = at4(grad), m4 = at4(m), v4 = at4(v), c4 = at4((const __bf16 *)t.copy);
    const unsigned key = adamw_mix(A.key + tensor);

    auto load = [&](int b, AdamwLoaded<P, G, BITS> &x) {
        const int64_t first = begin + b * 1024, i = first + 4 * lane;
        if (!WHOLE && first >= n) return;
        load4<WHOLE>(p, i, n, p4, x.p);
        load4<WHOLE>(grad, i, n, g4, x.g);
        load4<WHOLE>(m, i, n, m4, x.m);
        load4<WHOLE>(v, i, n, v4, x.v);
        if constexpr (BITS == 8) {
            x.mu = t.m_unit[first / 256];
            x.vu = t.v_unit[first / 256];
        }
    };
    auto update = [&](int b, AdamwLoaded<P, G, BITS> &x) {
        const int64_t first = begin + b * 1024, i = first + 4 * lane;
        if (!WHOLE && first >= n) return;
        float q[4];
        if constexpr (BITS == 32) {
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const AdamwElement o = adamw_element(A, (float)x.p[e], (float)x.g[e], x.m[e], x.v[e]);
                q[e] = o.p;
                x.m[e] = o.m;
                x.v[e] = o.v;
            }
        } else {
            const int64_t block = first / 256;
            float mx[4], vx[4];
            unsigned mtop = 0, vtop = 0;  // words of the largest magnitudes
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float m0 = code_value<3>(x.m[e] & 127u) * x.mu;
                const AdamwElement o = adamw_element(A, (float)x.p[e], (float)x.g[e], x.m[e] & 128u ? -m0 : m0, code_value<4>(x.v[e]) * x.vu);
                q[e] = o.p;
                const bool in = WHOLE || i + e < n;
                mx[e] = in ? o.m : 0.0f;
                vx[e] = in ? o.v : 0.0f;
                const unsigned mw = __float_as_uint(mx[e]) & 0x7fffffffu, vw = __float_as_uint(vx[e]) & 0x7fffffffu;
                mtop = mtop > mw ? mtop : mw;
                vtop = vtop > vw ? vtop : vw;
            }
            mtop = wave_max(mtop);
            vtop = wave_max(vtop);
            float minv, vinv;
            float mnew = block_unit<3>(mtop, minv), vnew = block_unit<4>(vtop, vinv);
            const unsigned bkey = adamw_mix(adamw_mix(key + (unsigned)block) + (unsigned)(block >> 32));
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const unsigned h = adamw_mix(bkey + (4 * lane + e) * 0x9E3779B9u);
                x.m[e] = (unsigned char)(code_of<3>(fabsf(mx[e]) * minv, h >> 16) | (mx[e] < 0.0f ? 128u : 0u));
                const float z = vx[e] * vinv;
                const unsigned c = code_of<4>(z, h & 0xffffu);
                x.v[e] = (unsigned char)(z > 0.0f && c == 0 ? 1u : c);
            }
            if (mtop >= 0x7f800000u) {
                mnew = __uint_as_float(0x7fc00000u);
#pragma unroll
                for (int e = 0; e < 4; e++) x.m[e] = 0;
            }
            if (vtop >= 0x7f800000u) {
                vnew = __uint_as_float(0x7fc00000u);
#pragma unroll
                for (int e = 0; e < 4; e++) x.v[e] = 0;
            }
            if (lane == 0) {
                t.m_unit[block] = mnew;
                t.v_unit[block] = vnew;
            }
        }
        store4<WHOLE>(m, i, n, m4, x.m);
        store4<WHOLE>(v, i, n, v4, x.v);
#pragma unroll
        for (int e = 0; e < 4; e++) x.p[e] = (P)q[e];
        store4<WHOLE>(p, i, n, p4, x.p);
        if (t.copy) {
            if (A.copy_f16) {
                _Float16 c[4];
#pragma unroll
                for (int e = 0; e < 4; e++) c[e] = (_Float16)q[e];
                store4<WHOLE>((_Float16 *)t.copy, i, n, c4, c);
            } else {
                __bf16 c[4];
#pragma unroll
                for (int e = 0; e < 4; e++) c[e] = (__bf16)q[e];
                store4<WHOLE>((__bf16 *)t.copy, i, n, c4, c);
            }
        }
    };
    // the next block is on its way while one is computed
    AdamwLoaded<P, G, BITS> x[2];
    load(0, x[0]);
#pragma unroll
    for (int b = 0; b < BLOCKS; b++) {
        if (b + 1 < BLOCKS) load(b + 1, x[(b + 1) & 1]);
        update(b, x[b & 1]);
    }
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
    const int64_t begin = (int64_t)(blockIdx.x - A.first[lo]) * TA_CHUNK;
    typedef typename std::conditional<BITS == 8, unsigned char, float>::type State;
    const bool aligned = at4((P *)t.p) && at4((const G *)t.grad) && at4((State *)t.m) && at4((State *)t.v) && at4((const __bf16 *)t.copy);
    const unsigned tensor = (unsigned)(A.tensor0 + lo);
    int64_t first = begin + TG_UNIFORM((int)(threadIdx.x >> 6)) * 256;
    if (aligned && begin + TA_CHUNK <= t.n) return adamw_chunk<P, G, BITS, true, TA_CHUNK / 1024>(A, t, first, tensor);
    // a tensor's end: its whole blocks without conditions likewise
#pragma unroll 1
    for (int b = 0; b < TA_CHUNK / 1024; b++, first += 1024) {
        if (aligned && first + 256 <= t.n) adamw_chunk<P, G, BITS, true, 1>(A, t, first, tensor);
        else adamw_chunk<P, G, BITS, false, 1>(A, t, first, tensor);
    }
}

struct ReadStatesArgs {
    struct One { const unsigned char *m, *v; const float *m_unit, *v_unit; float *m_out, *v_out; int64_t n; } t[TA_TENSORS];
    unsigned first[TA_TENSORS + 1];
    int n;
};
template <bool WHOLE> __device__ __forceinline__ void adamw_read_chunk(const ReadStatesArgs::One &t, int64_t begin) {
    const int lane = threadIdx.x & 63, wave = TG_UNIFORM((int)(threadIdx.x >> 6));
    // all blocks are requested before the first is written
    constexpr int BLOCKS = TA_CHUNK / 1024;
    unsigned char mc[BLOCKS][4], vc[BLOCKS][4];
    float mu[BLOCKS], vu[BLOCKS];
    const bool m4 = at4(t.m), v4 = at4(t.v), mo4 = at4(t.m_out), vo4 = at4(t.v_out);
#pragma unroll
    for (int b = 0; b < BLOCKS; b++) {
        const int64_t first = begin + (b * 4 + wave) * 256, i = first + 4 * lane;
        if (!WHOLE && first >= t.n) continue;
        if (t.m_out) {
            mu[b] = t.m_unit[first / 256];
            load4<WHOLE>(t.m, i, t.n, m4, mc[b]);
        }
        if (t.v_out) {
            vu[b] = t.v_unit[first / 256];
            load4<WHOLE>(t.v, i, t.n, v4, vc[b]);
        }
    }
#pragma unroll
    for (int b = 0; b < BLOCKS; b++) {
        const int64_t first = begin + (b * 4 + wave) * 256, i = first + 4 * lane;
        if (!WHOLE && first >= t.n) continue;
        float x[4];
        if (t.m_out) {
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float v = code_value<3>(mc[b][e] & 127u) * mu[b];
                x[e] = mc[b][e] & 128u ? -v : v;
            }
            store4<WHOLE>(t.m_out, i, t.n, mo4, x);
        }
        if (t.v_out) {
#pragma unroll
            for (int e = 0; e < 4; e++) x[e] = code_value<4>(vc[b][e]) * vu[b];
            store4<WHOLE>(t.v_out, i, t.n, vo4, x);
        }
    }
}

__global__ void __launch_bounds__(256) adamw_read_kernel(ReadStatesArgs A) {
    int lo = 0, hi = A.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (A.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    const ReadStatesArgs::One &t = A.t[lo];
    const int64_t begin = (int64_t)(blockIdx.x - A.first[lo]) * TA_CHUNK;
    if (begin + TA_CHUNK <= t.n && at4(t.m) && at4(t.v) && at4(t.m_out) && at4(t.v_out)) adamw_read_chunk<true>(t, begin);
    else adamw_read_chunk<false>(t, begin);
}
