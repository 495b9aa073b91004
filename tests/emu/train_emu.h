// CPU stand-in for what the training kernels use beyond hip_emu.h: waves that exchange values, matrix instructions, loads to LDS
// that arrive when they are waited for, LDS reads within the kernel's array.  Test scaffolding, like hip_emu.h.
#pragma once
#include "hip_emu.h"

typedef float emu_f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned emu_u32x4 __attribute__((ext_vector_type(4)));
typedef short emu_s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 emu_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 emu_f16x8 __attribute__((ext_vector_type(8)));

struct uint2 { unsigned x, y; };
static inline uint2 make_uint2(unsigned x, unsigned y) { return uint2{x, y}; }
static inline unsigned __float_as_uint(float f) { unsigned u; memcpy(&u, &f, 4); return u; }
static inline float __uint_as_float(unsigned u) { float f; memcpy(&f, &u, 4); return f; }
template <class T> static inline T min(T a, T b) { return a < b ? a : b; }

// the kernel's LDS array; reads and loads outside it are counted by emu_errors()
void emu_lds_range(const char *base, size_t bytes);
const char *emu_lds_check(const char *p, size_t bytes);
// 16 bytes to lds + 16 * lane from descriptor + offset (zeros beyond its end), when waited for
void emu_load_to_lds(uintptr_t lds, unsigned offset, emu_u32x4 descriptor);
void emu_wait_loads(int newest);
// D = first second^T: lane l holds rows 4*(l/16) .. +3 of column l % 16
emu_f32x4 emu_mfma_bf16(emu_bf16x8 first, emu_bf16x8 second, emu_f32x4 c);
emu_f32x4 emu_mfma_f16(emu_f16x8 first, emu_f16x8 second, emu_f32x4 c);
emu_f32x4 emu_mfma_f32(float first, float second, emu_f32x4 c);
emu_s16x4 emu_read_transposed(const char *p);
unsigned emu_wave_max(unsigned v);
// sum over the groups of `lanes` lanes, pairs first: every lane gets the same bits
float emu_lanes_sum(float x, int lanes);
// 4-bit codes in sixteenths; word s of a lane in row q of 16 lanes from word q of the lane in row s
float emu_code_to_float(unsigned c);
emu_u32x4 emu_exchange_words(emu_u32x4 w);
// all lanes of the wave have come here
void emu_wave_fence();
