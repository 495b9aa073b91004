// Element types, activations and small helpers of the cleartext training kernels.
#pragma once
#ifndef CKKSMI_EMULATE
#include <hip/hip_runtime.h>
#endif

#include <cstdint>

#include "../../include/ckksmi_train.h"

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// What the kernels use of the machine beyond plain HIP; with CKKSMI_EMULATE the tests' stand-in on the CPU has it instead
#ifdef CKKSMI_EMULATE
typedef uintptr_t LdsAddress;
typedef const char *LdsPointer;
#define TG_LDS(array) emu_lds_range(array, sizeof(array))
#define TG_OPAQUE(x) (void)0
#define TG_SCHEDULED() (void)0
#define TG_UNIFORM(x) (x)
#else
typedef unsigned LdsAddress;
typedef const __attribute__((address_space(3))) char *LdsPointer;
#define TG_LDS(array) (void)0
#define TG_OPAQUE(x) asm volatile("" : "+v"(x))  // the compiler knows nothing of x's value
#define TG_SCHEDULED() __builtin_amdgcn_sched_barrier(0)  // no instruction moves across
#define TG_UNIFORM(x) __builtin_amdgcn_readfirstlane(x)
#endif

inline size_t element_bytes(int dtype) { return dtype == CKKSMI_F32 ? 4 : 2; }

// 8 consecutive elements, 16-byte aligned
template <class T> struct Oct { T v[8]; };
template <class T> __device__ __forceinline__ void load_oct(const T *p, float (&x)[8]) {
    Oct<T> o;
    u32x4 *w = (u32x4 *)&o;
    const u32x4 *s = (const u32x4 *)p;
    w[0] = s[0];
    if constexpr (sizeof(T) == 4) w[1] = s[1];
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] = (float)o.v[e];
}
template <class T> __device__ __forceinline__ void store_oct(T *p, const float (&x)[8]) {
    Oct<T> o;
#pragma unroll
    for (int e = 0; e < 8; e++) o.v[e] = (T)x[e];
    const u32x4 *w = (const u32x4 *)&o;
    u32x4 *d = (u32x4 *)p;
    d[0] = w[0];
    if constexpr (sizeof(T) == 4) d[1] = w[1];
}

// 32-bit values kept in 24 bits: the upper 16 of their words in one plane, the next 8 (rounded to nearest even) in another
__device__ __forceinline__ void store_oct24(uint16_t *hi, uint8_t *lo, const float (&x)[8]) {
    u32x4 h;
    unsigned l[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; e++) {
        unsigned w = __float_as_uint(x[e]);
        w += 0x7fu + ((w >> 8) & 1u);
        if (e % 2 == 0) h[e / 2] = w >> 16;
        else h[e / 2] |= w & 0xffff0000u;
        l[e / 4] |= ((w >> 8) & 0xffu) << (8 * (e % 4));
    }
    *(u32x4 *)hi = h;
    *(uint2 *)lo = make_uint2(l[0], l[1]);
}
__device__ __forceinline__ void load_oct24(const uint16_t *hi, const uint8_t *lo, float (&x)[8]) {
    const u32x4 h = *(const u32x4 *)hi;
    const uint2 l2 = *(const uint2 *)lo;
    const unsigned l[2] = {l2.x, l2.y};
#pragma unroll
    for (int e = 0; e < 8; e++)
        x[e] = __uint_as_float((e % 2 ? h[e / 2] & 0xffff0000u : h[e / 2] << 16) | ((l[e / 4] >> (8 * (e % 4))) & 0xffu) << 8);
}

struct Activation { int kind; float c[4]; };

// act(g) in 32 bits (the same bits as act_both's: an answer does not depend on whether the pass saves)
__device__ __forceinline__ float act_value(const Activation &A, float g) {
    switch (A.kind) {
        case CKKSMI_ACT_POLY: return ((A.c[3] * g + A.c[2]) * g + A.c[1]) * g + A.c[0];
        case CKKSMI_ACT_RELU: return g < 0.0f ? 0.0f : g;  // (a NaN stays one)
        case CKKSMI_ACT_SILU: return g * (1.0f / (1.0f + expf(-g)));
        default: return g * (0.5f * (1.0f + erff(g * 0.70710678f)));
    }
}
// act(g) and its derivative
__device__ __forceinline__ void act_both(const Activation &A, float g, float &a, float &da) {
    switch (A.kind) {
        case CKKSMI_ACT_POLY:
            a = ((A.c[3] * g + A.c[2]) * g + A.c[1]) * g + A.c[0];
            da = (3.0f * A.c[3] * g + 2.0f * A.c[2]) * g + A.c[1];
            return;
        case CKKSMI_ACT_RELU:
            a = g < 0.0f ? 0.0f : g;
            da = g > 0.0f ? 1.0f : 0.0f;
            return;
        case CKKSMI_ACT_SILU: {
            const float q = 1.0f / (1.0f + expf(-g));
            a = g * q;
            da = q * (1.0f + g * (1.0f - q));
            return;
        }
        default: {
            const float q = 0.5f * (1.0f + erff(g * 0.70710678f));
            a = g * q;
            da = q + g * expf(-0.5f * g * g) * 0.39894228f;
            return;
        }
    }
}
