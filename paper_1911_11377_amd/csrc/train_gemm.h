// Matrix products of the gated feed-forward block on the matrix cores.
//
//     C[m][n] = sum over k of A(m, k) * B(n, k)
//
// for the block's operand orders.  An operand "along k" has its k indices side by side in memory (x, weights of the forward
// pass); one "along rows" has its rows side by side (weights of the backward pass, both operands of the weights' gradients).
//
// Tiles.  A workgroup computes BM x BN results.  Both operands' tiles go from memory to LDS without registers in between (16 bytes a
// lane), some steps ahead of their use.  Lanes whose row, column or k index lies beyond the operand are pointed past the end
// of the load's descriptor and bring zeros, so no tile needs a case of its own.
//
// Lane layout: v_mfma_f32_16x16x32 (16 bits) or four v_mfma_f32_16x16x4 (32 bits) take 16 bytes of each operand a lane:
// row l % 16, k chunk l / 16.  B is the first operand, so lane l holds the results of A's row l % 16 and of B's rows
// 4*(l/16) .. +3.  The B rows of two fragments are taken so that a lane's results of both are 8 neighbouring columns.
//   along k    : LDS row r holds its 16-byte chunks at (chunk ^ swizzle(r)); a fragment is one ds_read_b128.
//   along rows : LDS row k holds the tile's rows; 16-bit fragments are two ds_read_b64_tr_b16 (a group of 16 lanes reads
//                4 k x 16 rows and gets them transposed), 32-bit ones four ds_read_b32.
#pragma once
#include "train_types.h"

#define TG_OUTSIDE 0x80000000u  // a lane offset beyond every descriptor's end

enum { EPI_GATE = 0, EPI_STORE = 1, EPI_DHID = 2 };

// What the forward pass saves and the backward pass reads: act(g) and u act'(g), in 32 bits where the weights' gradients are f32.
// 16-bit gradients need them in 24 bits only: their roundings to 16 bits are then dg's, du's and h's own and no others
// (kept in 16 bits, act(g) and u act'(g) would add as much again)
struct Kept {
    char *a, *da;            // upper 16 bits, or the values
    uint8_t *a_low, *da_low; // 8 bits below; null: 32 bits are kept
};

// What happens to 8 neighbouring results of a row
struct EpiArgs {
    void *o0, *o1;         // GATE: h; STORE: the result; DHID: dg, du
    int arrays;            // GATE, DHID: 16-bit arrays that o0 and o1 each are (store_parts)
    size_t array_bytes;    // from one of them to the next
    Kept kept;             // GATE: to be written (a null: nothing is kept); DHID: to be read
    size_t ldo;            // elements, all of them
    int N;                 // columns
    int f32_out;           // STORE: the result is f32 whatever the operands
    int accumulate;        // STORE
    int whole;             // 8 columns may be stored at once: 16-byte aligned rows of at least the next multiple of 8
    Activation act;
};

#define TG_SOURCES 5
struct GemmProblem {
    const char *a[TG_SOURCES], *b[TG_SOURCES];  // STORE adds nsrc products, A0 B0 + A1 B1 + ..; GATE has two B's on one A
    size_t lda, ldb;          // bytes from one row (along k) or one k index (along rows) to the next
    int M, N, K;
    int nsrc;
    int tiles_m, tiles_n;
    float *part;              // k axis in parts: [splits][values][M][ld_part]
    size_t ld_part;
    EpiArgs epi;
};

#define TG_PROBLEMS 3
struct GemmArgs {
    GemmProblem p[TG_PROBLEMS];
    int first[TG_PROBLEMS + 1];  // tiles of the problems before
    int n_problems;
    int splits;                  // parts of the k axis, joined by gemm_join_kernel
};

// x rounded to T; with more arrays also x in three bf16 parts, each the rounding of what the ones before left: 24 bits over the whole range of
// f32.  For bf16 the rounded x is the first part, for f16 (whose range would cut small and large parts off) it is none of them
template <class T> __device__ __forceinline__ void store_parts(const EpiArgs &E, void *o, size_t at, const float (&x)[8]) {
    store_oct((T *)o + at, x);
    if constexpr (sizeof(T) == 2) {
        float r[8];
#pragma unroll
        for (int e = 0; e < 8; e++) r[e] = x[e];
        for (int p = 1; p < E.arrays; p++) {
            if (p > 1 || __is_same(T, __bf16))
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float part = (float)(__bf16)r[e];
                    r[e] = fabsf(part) <= 3.4e38f ? r[e] - part : 0.0f;  // what is not finite is in its first part alone
                }
            store_oct((__bf16 *)((char *)o + p * E.array_bytes) + at, r);
        }
    }
}
template <class T> __device__ __forceinline__ void store_kept(char *p, uint8_t *low, size_t at, const float (&x)[8]) {
    if (sizeof(T) == 4 || !low) store_oct((float *)p + at, x);
    else store_oct24((uint16_t *)p + at, low + at, x);
}
template <class T> __device__ __forceinline__ void load_kept(const char *p, const uint8_t *low, size_t at, float (&x)[8]) {
    if (sizeof(T) == 4 || !low) load_oct((const float *)p + at, x);
    else load_oct24((const uint16_t *)p + at, low + at, x);
}

template <class T, int EPI>
__device__ __forceinline__ void epilogue8(const EpiArgs &E, size_t m, int n, float (&v0)[8], float (&v1)[8]) {
    const size_t at = m * E.ldo + n;
    // columns that pad a row are zeros: they meet the zeros that pad the next product's other operand, and what an infinite row gives there is NaN
    if constexpr (EPI != EPI_STORE)
        if (n + 8 > E.N)
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (n + e >= E.N) v0[e] = v1[e] = 0.0f;
    if constexpr (EPI == EPI_GATE) {
        float h[8];
        if (E.kept.a) {
            float a[8], da[8];
#pragma unroll
            for (int e = 0; e < 8; e++) {
                act_both(E.act, v0[e], a[e], da[e]);
                da[e] *= v1[e];
                h[e] = a[e] * v1[e];
            }
            store_kept<T>(E.kept.a, E.kept.a_low, at, a);
            store_kept<T>(E.kept.da, E.kept.da_low, at, da);
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++) h[e] = act_value(E.act, v0[e]) * v1[e];
        }
        store_parts<T>(E, E.o0, at, h);
    } else if constexpr (EPI == EPI_DHID) {
        float a[8], da[8];
        load_kept<T>(E.kept.a, E.kept.a_low, at, a);
        load_kept<T>(E.kept.da, E.kept.da_low, at, da);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            da[e] *= v0[e];
            a[e] *= v0[e];
        }
        store_parts<T>(E, E.o0, at, da);
        store_parts<T>(E, E.o1, at, a);
    } else {
        float r[8];
        if (E.f32_out || sizeof(T) == 4) {
            float *o = (float *)E.o0 + at;
            if (E.whole) {
                if (E.accumulate) load_oct(o, r);
#pragma unroll
                for (int e = 0; e < 8; e++) r[e] = E.accumulate ? r[e] + v0[e] : v0[e];
                store_oct(o, r);
            } else {
                for (int e = 0; e < 8; e++)
                    if (n + e < E.N) o[e] = E.accumulate ? o[e] + v0[e] : v0[e];
            }
        } else {
            T *o = (T *)E.o0 + at;
            if (E.whole) {
                if (E.accumulate) load_oct(o, r);
#pragma unroll
                for (int e = 0; e < 8; e++) r[e] = E.accumulate ? r[e] + v0[e] : v0[e];
                store_oct(o, r);
            } else {
                for (int e = 0; e < 8; e++)
                    if (n + e < E.N) o[e] = (T)(E.accumulate ? (float)o[e] + v0[e] : v0[e]);
            }
        }
    }
}

// ---- operand tiles, SB bytes of k deep (128 or 64)
// swizzle of an LDS row's 16-byte chunks, so that the lanes of a fragment read spread over the banks.  Fragment rows:
// A takes 16 neighbouring rows; B takes rows 8*(i/4) + i%4 (+ 4 for the second fragment of a pair), i = lane % 16
template <bool IS_B, int SB> __device__ __forceinline__ int swizzle_k(int row) {
    if constexpr (SB == 64) return IS_B ? (row >> 3) & 3 : (row >> 2) & 3;
    return IS_B ? ((row >> 1) & 1) | ((row >> 3) & 3) << 1 : (row >> 1) & 7;
}
template <bool IS_B, int ES, int R> __device__ __forceinline__ int swizzle_rows(int k) {
    constexpr int chunks = R * ES / 16;  // of an LDS row: the swizzle stays among them
    const int q = (k >> 2) & 3;
    if constexpr (ES == 2) return (IS_B ? (k & 3) << 2 : ((k & 3) | ((k >> 3) & 1) << 2) << 1) & (chunks - 1);
    return (IS_B ? (q & 1) | (q >> 1) << 3 : q << 2) & (chunks - 1);
}

// 16 bytes a lane from a descriptor's memory to LDS: lane l's to lds + 16 l.  In assembly, so that the compiler, which takes every
// such load for a write to all of the LDS, does not wait for it before it reads the other stage: tile_barrier() waits.
// (No vector register is written by it.  The load takes its LDS address from m0 and has to stand one wait state behind the write of m0:
// the compiler fills none in inside a block.)
#ifdef CKKSMI_EMULATE
#define load_to_lds emu_load_to_lds
#define mfma_bf16 emu_mfma_bf16
#define mfma_f16 emu_mfma_f16
#define mfma_f32 emu_mfma_f32
static inline u32x4 descriptor(const char *p) { return u32x4{(unsigned)(uintptr_t)p, (unsigned)((uintptr_t)p >> 32), 0x7ffffff0u, 0}; }
template <int N> static inline void wait_loads() { emu_wait_loads(N); }
static inline void wave_barrier() { __syncthreads(); }
static inline void tile_barrier() { emu_wait_loads(0); __syncthreads(); }
static inline LdsAddress lds_address(const char *p) { return (uintptr_t)p; }
static inline LdsPointer lds_pointer(LdsAddress a) { return (const char *)a; }
static inline u32x4 lds_read16(LdsPointer p) { return *(const u32x4 *)emu_lds_check(p, 16); }
static inline unsigned lds_read4(LdsPointer p) { return *(const unsigned *)emu_lds_check(p, 4); }
static inline s16x4 lds_read_transposed(LdsPointer p) { return emu_read_transposed(emu_lds_check(p, 8)); }
#else
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 is one of the compiler's reserved registers: no value of its own lives there across the block)
__device__ __forceinline__ void load_to_lds(unsigned lds, unsigned offset, u32x4 descriptor) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(descriptor) : "memory", "m0");
}
#pragma clang diagnostic pop
#define mfma_bf16(a, b, c) __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0)
#define mfma_f16(a, b, c) __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0)
#define mfma_f32(a, b, c) __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0)
__device__ __forceinline__ u32x4 descriptor(const char *p) {
    const uint64_t a = (uint64_t)p;
    return u32x4{(unsigned)a, (unsigned)(a >> 32) & 0xffffu, 0x7ffffff0u, 0x00027000u};
}
// All but the wave's newest N loads have arrived
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wave_barrier() { asm volatile("s_barrier" ::: "memory"); }
// Every wave's loads to LDS have arrived, and every wave has read what it read before
__device__ __forceinline__ void tile_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ LdsAddress lds_address(const char *p) { return (unsigned)(uintptr_t)(LdsPointer)p; }
__device__ __forceinline__ LdsPointer lds_pointer(LdsAddress a) { return (LdsPointer)(uintptr_t)a; }
__device__ __forceinline__ u32x4 lds_read16(LdsPointer p) { return *(const __attribute__((address_space(3))) u32x4 *)p; }
__device__ __forceinline__ unsigned lds_read4(LdsPointer p) { return *(const __attribute__((address_space(3))) unsigned *)p; }
// a group of 16 lanes, lane i at 4 values of row i / 4: lane i gets the rows' values i
__device__ __forceinline__ s16x4 lds_read_transposed(LdsPointer p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p);
}
#endif

// Loads of one operand's tiles of R rows: what a lane needs to know, found once
template <class T, int R, int SB, bool ALONG_ROWS, bool IS_B, int WAVES, bool TWO>
struct TileLoad {
    static constexpr int ES = sizeof(T), EPC = 16 / ES, KSTEP = SB / ES;
    static constexpr int BYTES = R * SB;
    static constexpr int NI = BYTES / 1024 / WAVES;  // load instructions of a wave
    static constexpr int READS = !ALONG_ROWS ? 1 : ES == 2 ? 2 : 4;  // LDS reads of a fragment
    static_assert(NI * WAVES * 1024 == BYTES, "whole instructions");
    unsigned off[NI];  // byte offset of the lane's 16 bytes from the tile's first
    int kc[NI];        // their (first) k index within the step

    __device__ __forceinline__ void init(int wave, int lane, size_t ld, int rows_left) {
#pragma unroll
        for (int it = 0; it < NI; it++) {
            const int s = it * WAVES + wave;
            if constexpr (!ALONG_ROWS) {
                constexpr int CPR = SB / 16;  // chunks of an LDS row
                const int row = s * (64 / CPR) + lane / CPR, c = (lane % CPR) ^ swizzle_k<IS_B, SB>(row);
                const int mem_row = TWO && row >= R / 2 ? row - R / 2 : row;
                off[it] = mem_row < rows_left ? (unsigned)(mem_row * ld + c * 16) : TG_OUTSIDE;
                kc[it] = c * EPC;
            } else {
                constexpr int LPR = R * ES / 16, KPI = 64 / LPR;
                const int k = s * KPI + lane / LPR, c = (lane % LPR) ^ swizzle_rows<IS_B, ES, R>(k);
                off[it] = c * EPC < rows_left ? (unsigned)(k * ld + c * 16) : TG_OUTSIDE;
                kc[it] = k;
            }
        }
    }
    // instruction `it` of the tile at p0 (TWO: its second half at p1), whose first k_left k indices exist
    __device__ __forceinline__ void issue(LdsAddress lds, int wave, int it, const char *p0, const char *p1, int k_left) const {
        const unsigned o = k_left >= KSTEP || kc[it] < k_left ? off[it] : TG_OUTSIDE;
        load_to_lds(lds + (it * WAVES + wave) * 1024, o, descriptor(TWO && it >= NI / 2 ? p1 : p0));
    }
    // A lane's 16 bytes of the fragment whose first row is row0 (IS_B: of the pair's fragment `half`), sub-step kk (0: the first 64 bytes of k,
    // 1: the next): where they begin in the tile
    static __device__ __forceinline__ unsigned address(int row0, int half, int kk, int lane) {
        const int i = lane & 15, q = lane >> 4;
        if constexpr (!ALONG_ROWS) {
            const int row = IS_B ? row0 + 8 * (i >> 2) + 4 * half + (i & 3) : row0 + i;
            return row * SB + (((4 * kk + q) ^ swizzle_k<IS_B, SB>(row)) << 4);
        } else if constexpr (ES == 2) {
            // for the transposing read: k index i / 4 of the group's four, rows 4*(i % 4) .. +3 of the fragment's sixteen
            const int a = i & 3, row = IS_B ? row0 + 8 * a + 4 * half : row0 + 4 * a, k = 32 * kk + 8 * q + (i >> 2);
            return k * (R * ES) + (((row >> 3) ^ swizzle_rows<IS_B, ES, R>(k)) << 4) + (row & 4) * 2;
        } else {
            const int row = IS_B ? row0 + 8 * (i >> 2) + 4 * half + (i & 3) : row0 + i, k = 16 * kk + 4 * q;
            return k * (R * ES) + (((row >> 2) ^ swizzle_rows<IS_B, ES, R>(k)) << 4) + (row & 3) * 4;
        }
    }
    // ... and what is there (the swizzle is the same for all that is read)
    static __device__ __forceinline__ u32x4 read(LdsPointer p) {
        u32x4 f;
        if constexpr (!ALONG_ROWS) f = lds_read16(p);
        else if constexpr (ES == 2) {
            s16x4 h[2];
#pragma unroll
            for (int j = 0; j < 2; j++) h[j] = lds_read_transposed(p + j * 4 * R * ES);
            __builtin_memcpy(&f, h, 16);
        } else
#pragma unroll
            for (int j = 0; j < 4; j++) f[j] = lds_read4(p + j * R * ES);
        return f;
    }
    static __device__ __forceinline__ u32x4 fragment(const char *tile, int row0, int half, int kk, int lane) {
        return read((LdsPointer)tile + address(row0, half, kk, lane));
    }
};

template <class T> __device__ __forceinline__ f32x4 mma(const u32x4 &first, const u32x4 &second, f32x4 c) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 4; j++) c = mfma_f32(__uint_as_float(first[j]), __uint_as_float(second[j]), c);
        return c;
    } else if constexpr (__is_same(T, __bf16)) {
        return mfma_bf16(__builtin_bit_cast(bf16x8, first), __builtin_bit_cast(bf16x8, second), c);
    } else {
        return mfma_f16(__builtin_bit_cast(f16x8, first), __builtin_bit_cast(f16x8, second), c);
    }
}

// Tiles in the order in which their operands are shared: workgroups reach the 8 XCDs in turn, so each XCD takes a run of
// neighbouring tiles, and runs go down 8 tile rows before they move to the next tile column
__device__ __forceinline__ int xcd_order(int wg, int total) {
    const int per = total / 8, rest = total % 8, x = wg % 8, i = wg / 8;
    return x * per + (x < rest ? x : rest) + i;
}

// A workgroup's tile and its walk along the sources' k axes
template <class T, int BM, int BN, bool A_ROWS, bool B_ROWS, int EPI, class LA, class LB, int EVERY>
struct TileWalk {
    static constexpr bool GATE = EPI == EPI_GATE;
    const GemmProblem *P;
    int m0, n0;
    LA la;
    LB lb;
    int per_src, s0, s1, src, step;  // step: the next one to be issued, within its source
    size_t a_step, b_step, a_tile, b_tile;
    const char *pa, *pb, *pb1;
    int wave;

    __device__ __forceinline__ TileWalk(const GemmArgs &G, int wave_, int lane, int group) : wave(wave_) {
        int tile = xcd_order(blockIdx.x, gridDim.x), pi = 0;
        while (pi + 1 < G.n_problems && tile >= G.first[pi + 1]) pi++;
        tile -= G.first[pi];
        P = &G.p[pi];
        constexpr int GROUP = 8;
        const int band = tile / (GROUP * P->tiles_n), in_band = tile % (GROUP * P->tiles_n);
        const int band_rows = min(GROUP, P->tiles_m - band * GROUP);
        m0 = (band * GROUP + in_band % band_rows) * BM;
        n0 = in_band / band_rows * (GATE ? BN / 2 : BN);
        la.init(wave, lane, P->lda, P->M - m0);
        lb.init(wave, lane, P->ldb, P->N - n0);
        // steps s0 .. s1 - 1 of the sources', one source behind the other
        per_src = (P->K + LA::KSTEP - 1) / LA::KSTEP;
        const int steps = per_src * P->nsrc;
        s0 = (int)((long long)steps * blockIdx.y / G.splits);
        s1 = (int)((long long)steps * (blockIdx.y + 1) / G.splits);
        a_step = A_ROWS ? LA::KSTEP * P->lda : LA::KSTEP * sizeof(T);
        b_step = B_ROWS ? LA::KSTEP * P->ldb : LA::KSTEP * sizeof(T);
        a_tile = A_ROWS ? (size_t)m0 * sizeof(T) : (size_t)m0 * P->lda;
        b_tile = B_ROWS ? (size_t)n0 * sizeof(T) : (size_t)n0 * P->ldb;
        src = 0;
        step = s0 + group;
        enter();
    }
    __device__ __forceinline__ void enter() {
        while (step >= per_src && src + 1 < P->nsrc) {
            step -= per_src;
            src++;
        }
        pa = P->a[src] + a_tile + step * a_step;
        pb = P->b[src] + b_tile + step * b_step;
        pb1 = GATE ? P->b[1] + b_tile + step * b_step : nullptr;
    }
    static constexpr int LOADS = LA::NI + LB::NI;
    // load instruction `l` of LOADS of the next step's tiles
    __device__ __forceinline__ void issue(LdsAddress lds, int l) const {
        const int k_left = P->K - step * LA::KSTEP;
        if (l < LA::NI) la.issue(lds, wave, l, pa, nullptr, k_left);
        else lb.issue(lds + LA::BYTES, wave, l - LA::NI, pb, pb1, k_left);
    }
    // moves on by EVERY steps
    __device__ __forceinline__ void advance() {
        step += EVERY;
        if (EPI == EPI_STORE && step >= per_src && src + 1 < P->nsrc) return enter();
        pa += EVERY * a_step;
        pb += EVERY * b_step;
        if constexpr (GATE) pb1 += EVERY * b_step;
    }
    __device__ __forceinline__ void issue_all(LdsAddress lds) {
#pragma unroll
        for (int l = 0; l < LOADS; l++) issue(lds, l);
        advance();
    }
    // first LDS row of a wave's fragment pair p of B; GATE: even pairs are of the gate's weights, odd ones of the other's
    template <int WN> static __device__ __forceinline__ int b_row(int wn, int p) { return GATE ? p % 2 * (BN / 2) + wn * (WN / 2) + p / 2 * 32 : wn * WN + 32 * p; }
};

// A wave's results to memory, 8 neighbouring columns at a time
template <class T, int EPI, int FM, int PAIRS, int WN>
__device__ __forceinline__ void write_tile(const GemmArgs &G, const GemmProblem &P, int m_wave, int n0, int wn, int lane, const f32x4 (&acc)[FM][2 * PAIRS]) {
    constexpr bool GATE = EPI == EPI_GATE;
    static_assert(!GATE || PAIRS % 2 == 0, "a wave holds the same columns of both products");
    const int i = lane & 15, q = lane >> 4;
#pragma unroll
    for (int f = 0; f < FM; f++) {
        const int m = m_wave + 16 * f + i;
        if (m >= P.M) continue;
        auto eight = [&](int p, float (&v)[8]) {
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = acc[f][2 * p + e / 4][e % 4];
        };
        float v0[8], v1[8];
        if constexpr (GATE) {
#pragma unroll
            for (int p = 0; p < PAIRS; p += 2) {
                const int n = n0 + wn * (WN / 2) + 16 * p + 8 * q;
                if (n >= P.N) continue;
                eight(p, v0);
                eight(p + 1, v1);
                if (G.splits > 1) {
                    float *o = P.part + ((size_t)blockIdx.y * 2 * P.M + m) * P.ld_part + n;
                    store_oct(o, v0);
                    store_oct(o + (size_t)P.M * P.ld_part, v1);
                } else
                    epilogue8<T, EPI>(P.epi, m, n, v0, v1);
            }
        } else {
#pragma unroll
            for (int p = 0; p < PAIRS; p++) {
                const int n = n0 + wn * WN + 32 * p + 8 * q;
                if (n >= P.N) continue;
                eight(p, v0);
                if (G.splits > 1) store_oct(P.part + ((size_t)blockIdx.y * P.M + m) * P.ld_part + n, v0);
                else epilogue8<T, EPI>(P.epi, m, n, v0, v0);
            }
        }
    }
}

// Large tiles, two LDS stages of 128 bytes of k.  A step's products come in four quarters (two halves of k, two halves of A's
// rows); while one quarter is formed, the next one's fragments come from LDS.  With the third quarter a wave has read all of
// its stage, and the other stage has arrived: the step's one barrier stands there, behind it the last quarter is formed while
// the next step's first fragments are read and the tiles of the step after that are requested into the stage just left.
// The requests stand between that quarter's products, not at once: a load instruction keeps the memory path busy for 16 cycles.
// Rows of 128 bytes a stage: with four stages of 64 bytes a row the loads reach half the rate (68 GB/s a compute unit against 128) and the
// forward product of 4096 rows, columns and indices took 147 us instead of 126.
// Bound by the matrix cores and what keeps them waiting at the barrier: 59 - 64 % of the cycles busy there (a library's product: 86 %).
// Measured, bf16, 16384 rows, 2048 -> 8192 -> 2048: gate with what is kept 1.26 ms (0.87 PFLOP/s; 1.07 GB written after the products,
// a quarter of the time), down 0.48 ms (1.15), dh 0.80 ms (0.69; 0.8 GB read and 0.54 GB written after the products), dx 0.86 ms
// (1.28), weights' gradients 1.31 ms (1.26); both products of 4096^3 330 - 337 us (1.23).
template <class T, int BM, int BN, int WM, int WN, bool A_ROWS, bool B_ROWS, int EPI>
__global__ void __launch_bounds__(64 * (BM / WM) * (BN / WN), 2) gemm_kernel(GemmArgs G) {
    constexpr int WAVES = (BM / WM) * (BN / WN), FM = WM / 16, PAIRS = WN / 32, SB = 128, HALF = FM / 2;
    typedef TileLoad<T, BM, SB, A_ROWS, false, WAVES, false> LA;
    typedef TileLoad<T, BN, SB, B_ROWS, true, WAVES, EPI == EPI_GATE> LB;
    typedef TileWalk<T, BM, BN, A_ROWS, B_ROWS, EPI, LA, LB, 1> Walk;
    constexpr int STAGE = LA::BYTES + LB::BYTES, LOADS = Walk::LOADS;
    __shared__ __attribute__((aligned(1024))) char stages[2 * STAGE];
    TG_LDS(stages);
    const int lane = threadIdx.x & 63, wave = TG_UNIFORM((int)(threadIdx.x >> 6));
    const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN);
    Walk w(G, wave, lane, 0);
    const int n = w.s1 - w.s0;

    f32x4 acc[FM][2 * PAIRS];
#pragma unroll
    for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < 2 * PAIRS; j++) acc[i][j] = f32x4{0, 0, 0, 0};
    u32x4 a[FM], b[2][2 * PAIRS];
    // Lane addresses in LDS, of the stage at hand (an LDS instruction's offset does not reach the other one; the addresses are kept from the
    // compiler, which would hold a set of registers for each).  Along k all fragments of a half step lie at constant distances,
    // along rows the halves do, and the swizzle gives each fragment its own address
    constexpr int NA = A_ROWS ? FM : 2, NB = !B_ROWS ? 2 : sizeof(T) == 2 ? PAIRS : 2 * PAIRS;
    const LdsAddress lds = lds_address(stages);
    LdsAddress at_a[NA], at_b[NB];
#pragma unroll
    for (int f = 0; f < NA; f++) at_a[f] = lds + (A_ROWS ? LA::address(wm + 16 * f, 0, 0, lane) : LA::address(wm, 0, f, lane));
#pragma unroll
    for (int f = 0; f < NB; f++) {
        const int p = NB == PAIRS ? f : f / 2, h = NB == PAIRS ? 0 : f % 2;
        at_b[f] = lds + LA::BYTES + (B_ROWS ? LB::address(Walk::template b_row<WN>(wn, p), h, 0, lane) : LB::address(Walk::template b_row<WN>(wn, 0), 0, f, lane));
    }
    auto move = [&](int by) {
#pragma unroll
        for (int f = 0; f < NA; f++) {
            at_a[f] += by;
            TG_OPAQUE(at_a[f]);
        }
#pragma unroll
        for (int f = 0; f < NB; f++) {
            at_b[f] += by;
            TG_OPAQUE(at_b[f]);
        }
    };
    constexpr int KHALF = LA::KSTEP / 2;  // k indices of a half step
    auto read_a = [&](int f, int kk) {
        a[f] = LA::read(lds_pointer(at_a[A_ROWS ? f : kk]) + (A_ROWS ? kk * KHALF * BM * (int)sizeof(T) : f * 16 * SB));
    };
    // B's fragments of a half step and the first half of A's; the second half of A's
    auto read_first = [&](int kk) {
#pragma unroll
        for (int p = 0; p < PAIRS; p++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const LdsPointer base = lds_pointer(at_b[!B_ROWS ? kk : NB == PAIRS ? p : 2 * p + h]);
                const int row = Walk::template b_row<WN>(0, p) - Walk::template b_row<WN>(0, 0);
                b[kk][2 * p + h] = LB::read(base + (!B_ROWS ? (row + 4 * h) * SB : kk * KHALF * BN * (int)sizeof(T) + (NB == PAIRS ? 8 * h : 0)));
            }
#pragma unroll
        for (int i = 0; i < HALF; i++) read_a(i, kk);
    };
    auto read_second = [&](int kk) {
#pragma unroll
        for (int i = HALF; i < FM; i++) read_a(i, kk);
    };
    // a quarter's products; among them the load instructions l0 .. l1 - 1 of a later step's tiles
    auto multiply = [&](int kk, int from, int l0, int l1, LdsAddress stage) {
#pragma unroll
        for (int i = 0; i < HALF; i++) {
#pragma unroll
            for (int j = 0; j < 2 * PAIRS; j++) acc[from + i][j] = mma<T>(b[kk][j], a[from + i], acc[from + i][j]);
#pragma unroll
            for (int l = l0; l < l1; l++)
                if ((l - l0) * HALF / (l1 - l0) == i) {
                    TG_SCHEDULED();
                    w.issue(stage, l);
                    TG_SCHEDULED();
                }
        }
    };
    // Requests run up to two steps past the last one: they bring zeros, or k indices of another part, to stages that nobody reads any more
    w.issue_all(lds);
    w.issue_all(lds + STAGE);
    wait_loads<LOADS>();
    wave_barrier();
    read_first(0);
    int other = STAGE;  // from the stage at hand to the other one
    LdsAddress stage = lds;
    for (int t = 0; t < n; t++) {
        read_second(0);
        multiply(0, 0, 0, 0, 0);
        read_first(1);
        multiply(0, HALF, 0, 0, 0);
        read_second(1);
        multiply(1, 0, 0, 0, 0);
        TG_SCHEDULED();  // the products of what was read stay before
        tile_barrier();
        move(other);
        read_first(0);
        multiply(1, HALF, 0, LOADS, stage);
        w.advance();
        stage += other;
        other = -other;
    }
    wait_loads<0>();
    write_tile<T, EPI, FM, PAIRS, WN>(G, *w.P, w.m0 + wm, w.n0, wn, lane, acc);
}

// Small tiles, for products that are bound by latency: KG groups of waves share the k axis step by step, each with two LDS
// stages of 128 bytes of k of its own; group 0 adds up the groups' sums in their order.  One group where there are more tiles
// than compute units (three or four workgroups share one then) or no more than two steps.
// Measured: bf16, 333 rows of 517 -> 1021, gate 11 us (176 tiles, four groups; 128 x 128 in two parts and their join 18), weights'
// gradients of three parts each 17 us (360 tiles, one group; four groups 22); f32, 64 rows, 3136 x 256: 7.7 us (402 tiles; 11.7).
template <class T, int BM, int BN, int WM, int WN, int KG, bool A_ROWS, bool B_ROWS, int EPI>
__global__ void __launch_bounds__(64 * (BM / WM) * (BN / WN) * KG) gemm_small_kernel(GemmArgs G) {
    constexpr int WAVES = (BM / WM) * (BN / WN), FM = WM / 16, PAIRS = WN / 32, SB = 128;
    typedef TileLoad<T, BM, SB, A_ROWS, false, WAVES, false> LA;
    typedef TileLoad<T, BN, SB, B_ROWS, true, WAVES, EPI == EPI_GATE> LB;
    typedef TileWalk<T, BM, BN, A_ROWS, B_ROWS, EPI, LA, LB, KG> Walk;
    constexpr int STAGE = LA::BYTES + LB::BYTES;
    __shared__ __attribute__((aligned(1024))) char stages[KG * 2 * STAGE];
    TG_LDS(stages);
    const int lane = threadIdx.x & 63, wave_of_all = TG_UNIFORM((int)(threadIdx.x >> 6)), wave = wave_of_all % WAVES, group = wave_of_all / WAVES;
    char *const stage0 = stages + group * 2 * STAGE, *const stage1 = stage0 + STAGE;
    const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN);
    Walk w(G, wave, lane, group);

    f32x4 acc[FM][2 * PAIRS];
#pragma unroll
    for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < 2 * PAIRS; j++) acc[i][j] = f32x4{0, 0, 0, 0};
    auto multiply = [&](const char *st) {
        u32x4 b[2 * PAIRS];
#pragma unroll
        for (int kk = 0; kk < 2; kk++) {
#pragma unroll
            for (int p = 0; p < PAIRS; p++)
#pragma unroll
                for (int h = 0; h < 2; h++) b[2 * p + h] = LB::fragment(st + LA::BYTES, Walk::template b_row<WN>(wn, p), h, kk, lane);
#pragma unroll
            for (int i = 0; i < FM; i++) {
                const u32x4 a = LA::fragment(st, wm + 16 * i, 0, kk, lane);
#pragma unroll
                for (int j = 0; j < 2 * PAIRS; j++) acc[i][j] = mma<T>(b[j], a, acc[i][j]);
            }
        }
    };
    const int rounds = (w.s1 - w.s0 + KG - 1) / KG, own = (w.s1 - w.s0 - group + KG - 1) / KG;  // of the workgroup, of this group
    if (own > 0) w.issue_all(lds_address(stage0));
    for (int r = 0; r < rounds; r += 2) {
        tile_barrier();
        if (r + 1 < own) w.issue_all(lds_address(stage1));
        if (r < own) multiply(stage0);
        if (r + 1 < rounds) {
            tile_barrier();
            if (r + 2 < own) w.issue_all(lds_address(stage0));
            if (r + 1 < own) multiply(stage1);
        }
    }
    if constexpr (KG > 1) {
        static_assert((KG - 1) * BM * BN * 4 <= KG * 2 * STAGE, "the other groups' sums fit the stages");
        f32x4 *sums = (f32x4 *)stages;
        tile_barrier();
#pragma unroll
        for (int f = 0; f < FM; f++)
#pragma unroll
            for (int j = 0; j < 2 * PAIRS; j++)
                if (group) sums[(((group - 1) * FM + f) * 2 * PAIRS + j) * WAVES * 64 + wave * 64 + lane] = acc[f][j];
        tile_barrier();
        if (group) return;
#pragma unroll
        for (int g = 0; g < KG - 1; g++)
#pragma unroll
            for (int f = 0; f < FM; f++)
#pragma unroll
                for (int j = 0; j < 2 * PAIRS; j++) acc[f][j] += sums[((g * FM + f) * 2 * PAIRS + j) * WAVES * 64 + wave * 64 + lane];
    }
    write_tile<T, EPI, FM, PAIRS, WN>(G, *w.P, w.m0 + wm, w.n0, wn, lane, acc);
}

// Sum of the parts of a split k axis, always in the same order, and the epilogue.  Memory bounds it: 4 parts of 2048 x 1024 7 us (33.5 MB
// read and 4.2 MB written, 5.4 TB/s)
template <class T, int EPI>
__global__ void __launch_bounds__(256) gemm_join_kernel(GemmArgs G) {
    constexpr int VALUES = EPI == EPI_GATE ? 2 : 1;
    const GemmProblem &P = G.p[blockIdx.y];
    const size_t octs = P.ld_part / 8, id = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= octs * P.M) return;
    const size_t m = id / octs;
    const int n = (int)(id % octs) * 8;
    float v[2][8] = {};
    for (int s = 0; s < G.splits; s++)
#pragma unroll
        for (int w = 0; w < VALUES; w++) {
            float x[8];
            load_oct(P.part + (((size_t)s * VALUES + w) * P.M + m) * P.ld_part + n, x);
#pragma unroll
            for (int e = 0; e < 8; e++) v[w][e] = s ? v[w][e] + x[e] : x[e];
        }
    epilogue8<T, EPI>(P.epi, m, n, v[0], v[1]);
}

// Copies with rows padded to whole 16-byte chunks (zeros behind the last column), for operands whose rows do not begin on them: one launch for
// all of a call's, 5.5 us for the 2.7 MB of 333 rows of 517 -> 1021 -> 129.  SPLIT: f16 values as the sum of two bf16 ones (their 11 bits fit), the
// second array `split` bytes behind the first: 8.8 us for 2048 rows of 1024 and 1024
#define TG_COPIES 5  // of one call: x, three weight matrices, dy
struct CopyArgs {
    struct One { const char *src; char *dst; size_t ld_src, ld_dst; int cols, chunks; size_t rows, split; unsigned first; } c[TG_COPIES];
    int n;
    unsigned per;  // pieces of 256 chunks of 16 bytes that a workgroup takes
};
template <class T, bool SPLIT> __global__ void __launch_bounds__(256) pad_rows_kernel(CopyArgs A) {
    int i = 0;
    while (i + 1 < A.n && blockIdx.x >= A.c[i + 1].first) i++;
    const CopyArgs::One &C = A.c[i];
    constexpr int EPC = 16 / sizeof(T);
    for (unsigned j = 0; j < A.per; j++) {
        const size_t id = ((size_t)(blockIdx.x - C.first) * A.per + j) * 256 + threadIdx.x;
        if (id >= C.rows * C.chunks) return;
        // (most copies are small enough for a 32-bit division)
        const size_t r = id >> 32 ? id / C.chunks : (unsigned)id / (unsigned)C.chunks;
        const int c = (int)(id - r * C.chunks) * EPC;
        const T *s = (const T *)(C.src + r * C.ld_src) + c;
        u32x4 w;
        if (c + EPC <= C.cols) __builtin_memcpy(&w, s, 16);
        else {
            T v[EPC];
#pragma unroll
            for (int e = 0; e < EPC; e++) v[e] = c + e < C.cols ? s[e] : (T)0.0f;
            __builtin_memcpy(&w, v, 16);
        }
        char *const d = C.dst + r * C.ld_dst + (size_t)c * sizeof(T);
        if constexpr (SPLIT) {
            T v[EPC];
            __builtin_memcpy(&v, &w, 16);
            float x[EPC];
#pragma unroll
            for (int e = 0; e < EPC; e++) x[e] = (float)v[e];
            store_oct((__bf16 *)d, x);
#pragma unroll
            for (int e = 0; e < EPC; e++) x[e] -= (float)(__bf16)x[e];
            store_oct((__bf16 *)(d + C.split), x);
        } else
            *(u32x4 *)d = w;
    }
}
