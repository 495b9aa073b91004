// Device side of include/ckksmi_train.h: argument checks and launch sequences.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "device_call.h"
#include "train_adamw.h"
#include "train_gemm.h"
#include "train_rows.h"

namespace {

constexpr int64_t kMaxDim = 1 << 20, kMaxRows = 0x7fffffff - 256;
constexpr double kMaxThreads = 4294967295.0;  // of a launch, along x
constexpr int kMaxBlocks = (1 << 24) - 1;      // workgroups of 256 threads
#ifndef TG_COPY_BLOCKS
#define TG_COPY_BLOCKS (1 << 23)  // of a launch that copies operands: beyond, each takes several pieces (the tests' stand-in sets it)
#endif
constexpr int64_t kMaxNumel = (int64_t)kMaxBlocks * TA_CHUNK;

inline size_t round_up(size_t v, size_t to) { return (v + to - 1) / to * to; }
inline bool aligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
inline bool dtype_ok(int d) { return d == CKKSMI_F32 || d == CKKSMI_BF16 || d == CKKSMI_F16; }

// (Entry points copy the caller's structure before they check it: what was checked is what is used)
int check_ff(const ckksmi_gated_ff &f) {
    if (!dtype_ok(f.dtype) || (f.grad_dtype != f.dtype && f.grad_dtype != CKKSMI_F32) || f.act < CKKSMI_ACT_POLY || f.act > CKKSMI_ACT_GELU) return CKKSMI_EINVAL;
    if (f.rows < 0 || f.rows > kMaxRows) return CKKSMI_EINVAL;
    const int64_t d[3] = {f.d_in, f.d_hidden, f.d_out};
    for (int64_t v : d)
        if (v < 1 || v > kMaxDim) return CKKSMI_EINVAL;
    const int64_t ld[4] = {f.ld_x, f.ld_y, f.ld_dy, f.ld_dx}, least[4] = {f.d_in, f.d_out, f.d_out, f.d_in};
    for (int i = 0; i < 4; i++)
        if (ld[i] != 0 && (ld[i] < least[i] || ld[i] > kMaxDim)) return CKKSMI_EINVAL;
    return CKKSMI_OK;
}

// [a, a + na) and [b, b + nb) share a byte
inline bool overlap(const void *a, size_t na, const void *b, size_t nb) {
    if (!a || !b || !na || !nb) return false;
    const char *x = (const char *)a, *y = (const char *)b;
    return x < y + nb && y < x + na;
}

// A workspace handed out piece by piece (workspace_of() has counted the pieces)
struct Carve {
    char *base;
    size_t used = 0;
    explicit Carve(void *p) : base((char *)p) {}
    char *take(size_t bytes) {
        char *p = base + used;
        used += round_up(bytes, 256);
        return p;
    }
};

// one operand of a product: rows of `cols` elements, `ld` bytes apart
struct Matrix {
    const char *p;
    size_t ld;
};

struct FF {  // a call's sizes
    size_t es, ges, M, K, H, O, ldh;
    explicit FF(const ckksmi_gated_ff &f)
        : es(element_bytes(f.dtype)), ges(element_bytes(f.grad_dtype)), M((size_t)f.rows), K((size_t)f.d_in), H((size_t)f.d_hidden), O((size_t)f.d_out), ldh(round_up(H, 8)) {}
    size_t hidden_bytes() const { return round_up(M * ldh * es, 256); }
    bool fine() const { return es == 2 && ges == 4; }  // f32 gradients of 16-bit operands
    // then h, dg and du enter the weights' gradients as sums of three bf16 parts.  Arrays that each is kept in: rounded to its type, for bf16 the
    // first part too; and the products that the gradients are the sum of: x and dy are one bf16 value, or (f16) two
    int arrays(int dtype) const { return !fine() ? 1 : dtype == CKKSMI_BF16 ? 3 : 4; }
    int sources(int dtype) const { return !fine() ? 1 : dtype == CKKSMI_BF16 ? 3 : 5; }
    // what a forward pass saves: act(g), u act'(g) (4 bytes, or 2 + 1), h in its arrays
    size_t kept_bytes() const { return fine() ? round_up(M * ldh * 4, 256) : hidden_bytes(); }
    size_t low_bytes() const { return es == 2 && !fine() ? round_up(M * ldh, 256) : 0; }
    size_t saved_bytes(int dtype) const { return 2 * kept_bytes() + 2 * low_bytes() + arrays(dtype) * hidden_bytes(); }
    Kept kept(const void *saved) const {
        char *p = (char *)saved;
        uint8_t *low = (uint8_t *)p + 2 * kept_bytes();
        return low_bytes() ? Kept{p, p + kept_bytes(), low, low + low_bytes()} : Kept{p, p + kept_bytes(), nullptr, nullptr};
    }
    char *saved_h(const void *saved) const { return (char *)saved + 2 * kept_bytes() + 2 * low_bytes(); }
};
inline size_t ld_bytes(int64_t ld, size_t cols, size_t es) { return (ld ? (size_t)ld : cols) * es; }

Activation activation_of(const ckksmi_gated_ff &f) {
    Activation a;
    a.kind = f.act;
    memcpy(a.c, f.c, sizeof(a.c));
    return a;
}

// What a product's launch looks like: tile shape (an index of kTiles) and parts of the k axis
struct Shape { int tile, splits; };
struct TileShape { int bm, bn; };
constexpr TileShape kTiles[3] = {{256, 256}, {128, 128}, {32, 128}};
constexpr int kMaxSplits = 32;
// a k axis in parts: workgroups that the parts together may come to, and steps of 128 bytes that each has at least (128 x 128, 32 x 128)
constexpr int kParts[2] = {512, 384}, kPartSteps[2] = {4, 8};
constexpr double kMuchWork = 4e9;  // operations
#ifndef TG_ENOUGH_TILES
#define TG_ENOUGH_TILES 192  // three quarters of the compute units (the tests' stand-in sets it)
#endif

long long tiles_of(const GemmProblem &p, const TileShape &t, bool gate, GemmProblem *out) {
    const int cols = gate ? t.bn / 2 : t.bn;
    const int tm = (p.M + t.bm - 1) / t.bm, tn = (p.N + cols - 1) / cols;
    if (out) { out->tiles_m = tm; out->tiles_n = tn; }
    return (long long)tm * tn;
}

inline int k_steps(const GemmProblem &p, size_t es) { return (int)(((size_t)p.K * es + 127) / 128) * p.nsrc; }  // of 128 bytes

// Tile and parts of the k axis.  Measured, us of one pass against the best (bf16 unless said):
//   enough 256 x 256 tiles for three quarters of the compute units: those
//       (gate, 2048 rows, 1024 -> 4096: 256 x 256 0, 128 x 128 +0.5, 32 x 128 +16)
//   enough 128 x 128 tiles likewise: those, the k axis whole (dx, 16384 rows, 500 -> 200: whole 0, two parts +7); f32, which the matrix cores
//       bound rather than the operands' bytes, from two a compute unit on (weights' gradients, 500 rows of 2000 x 1000, 304 tiles: 32 x 128 -17 of 137;
//       whole passes, 32 x 128 first: 1500 rows of 1500 -> 1500 -> 1500 forward 209 and 265, backward 428 and 420; 512 rows of 2048 -> 2048 -> 2048 114
//       and 126, 227 and 235; 2048 rows of 1024 -> 4096 -> 1024 398 and 393, 838 and 797; 3000 rows of 512 -> 512 -> 512 52 and 63, 130 and 122)
//   few tiles of much work: 128 x 128 with the k axis in parts (2048 x 1024 from 4096: 4 parts 0, 2 parts +3, 32 x 128 whole +4, 256 x 256 in 4 parts +9)
//   else 32 x 128, in parts where that leaves compute units idle
//       (f32 gate, 1024 rows, 3136 -> 256: 2 parts 0, 4 and 8 parts +2; 128 x 128 in 8 parts +5, in 16 +11)
Shape choose(const GemmProblem *p, int n, bool gate, size_t es) {
    long long tiles[3] = {0, 0, 0};
    double flops = 0;
    for (int i = 0; i < n; i++) {
        for (int t = 0; t < 3; t++) tiles[t] += tiles_of(p[i], kTiles[t], gate, nullptr);
        flops += 2.0 * p[i].M * p[i].N * p[i].K * (gate ? 2 : p[i].nsrc);
    }
    for (long long &t : tiles) t = std::max(t, 1LL);
    const int steps = k_steps(p[0], es);
    auto parts = [&](int t) { return (int)std::max(1LL, std::min(std::min(kParts[t - 1] / tiles[t], (long long)steps / kPartSteps[t - 1]), (long long)kMaxSplits)); };
    if (es == 2 && tiles[0] >= TG_ENOUGH_TILES) return Shape{0, 1};
    if (tiles[1] >= (es == 2 ? TG_ENOUGH_TILES : 8 * TG_ENOUGH_TILES / 3)) return Shape{1, 1};
    if (es == 2 && flops > kMuchWork && p[0].M > 64) return Shape{1, parts(1)};
    return Shape{2, parts(2)};
}

size_t part_bytes(const GemmProblem &p, int splits, bool gate) {
    return splits > 1 ? (size_t)splits * (gate ? 2 : 1) * p.M * round_up(p.N, 8) * sizeof(float) : 0;
}

// At least part_bytes() of the product on p.M rows and on any number below: fewer rows are fewer tiles, which choose() gives more parts, so
// the need itself goes up and down with the rows.  Parts x tiles are kParts at most, a tile's results lie in bm x bn values
// (both factors of a gate's among them), and the parts' number is bounded by the k axis, which does not depend on the rows
size_t part_bytes_up_to(const GemmProblem &p, bool gate, size_t es) {
    auto most = [&](int t) {
        const size_t parts = std::min(k_steps(p, es) / kPartSteps[t - 1], kMaxSplits);
        const size_t of_tiles = (size_t)kParts[t - 1] * kTiles[t].bm * kTiles[t].bn * sizeof(float);
        return parts > 1 ? std::min(part_bytes(p, (int)parts, gate), of_tiles) : 0;
    };
    const bool much = es == 2 && 2.0 * p.M * p.N * p.K * (gate ? 2 : p.nsrc) > kMuchWork && p.M > 64;
    return std::max(much ? most(1) : 0, most(2));
}

// Workgroups of a product's launch, 0 where it would have more threads than a launch holds (256 a workgroup, 512 for tiles of 256 x 256;
// groups of 1024 only up to 256 workgroups)
long long workgroups_of(const GemmProblem *p, int n, bool gate, size_t es) {
    const Shape s = choose(p, n, gate, es);
    long long total = 0;
    for (int i = 0; i < n; i++) total += tiles_of(p[i], kTiles[s.tile], gate, nullptr);
    return (double)total * (s.tile == 0 ? 512 : 256) > kMaxThreads ? 0 : total;
}

// Up to TG_PROBLEMS products of one kind in a launch; `w` gives the memory for a split k axis
template <class T, bool A_ROWS, bool B_ROWS, int EPI>
void launch_gemm(ckksmi_ctx *c, GemmProblem *p, int n, Carve w, hipStream_t st) {
    constexpr bool gate = EPI == EPI_GATE;
    const Shape s = choose(p, n, gate, sizeof(T));
    GemmArgs G;
    memset(&G, 0, sizeof(G));
    int total = 0, join = 0;
    double flops = 0;
    for (int i = 0; i < n; i++) {
        G.first[i] = total;
        total += (int)tiles_of(p[i], kTiles[s.tile], gate, &p[i]);  // (fits_grids() has bounded it)
        p[i].ld_part = round_up(p[i].N, 8);
        if (s.splits > 1) p[i].part = (float *)w.take(part_bytes(p[i], s.splits, gate));
        G.p[i] = p[i];
        join = std::max(join, (int)(((size_t)p[i].M * p[i].ld_part / 8 + 255) / 256));
        flops += 2.0 * p[i].M * p[i].N * p[i].K * (gate ? 2 : p[i].nsrc);
    }
    G.first[n] = total;
    G.n_problems = n;
    G.splits = s.splits;
    const dim3 grid(total, s.splits);
    if constexpr (sizeof(T) == 2)
        if (s.tile == 0) KL(c, CKKSMI_K_GEMM, flops, (gemm_kernel<T, 256, 256, 128, 64, A_ROWS, B_ROWS, EPI>), grid, dim3(512), st, G);
    if (s.tile == 1) KL(c, CKKSMI_K_GEMM, flops, (gemm_kernel<T, 128, 128, 64, 64, A_ROWS, B_ROWS, EPI>), grid, dim3(256), st, G);
    // four groups of waves take a compute unit each: where there are more tiles than those, or few steps to share, one group a tile
    const bool groups = s.tile == 2 && total * s.splits <= 256 && k_steps(p[0], sizeof(T)) > 2 * s.splits;
    if (groups) KL(c, CKKSMI_K_GEMM, flops, (gemm_small_kernel<T, 32, 128, 16, 64, 4, A_ROWS, B_ROWS, EPI>), grid, dim3(1024), st, G);
    else if (s.tile == 2) KL(c, CKKSMI_K_GEMM, flops, (gemm_small_kernel<T, 32, 128, 16, 64, 1, A_ROWS, B_ROWS, EPI>), grid, dim3(256), st, G);
    if (s.splits > 1) KL(c, CKKSMI_K_GEMM_JOIN, flops, (gemm_join_kernel<T, EPI>), dim3(join, n), dim3(256), st, G);
}

GemmProblem product(Matrix a, Matrix b, size_t M, size_t N, size_t K) {
    GemmProblem p;
    memset(&p, 0, sizeof(p));
    p.a[0] = a.p; p.b[0] = b.p; p.lda = a.ld; p.ldb = b.ld;
    p.M = (int)M; p.N = (int)N; p.K = (int)K; p.nsrc = 1;
    return p;
}

void store_to(GemmProblem &p, void *out, size_t ld_elements, int out_dtype, bool accumulate) {
    const size_t es = element_bytes(out_dtype);
    p.epi.o0 = out; p.epi.ldo = ld_elements; p.epi.N = p.N; p.epi.f32_out = out_dtype == CKKSMI_F32; p.epi.accumulate = accumulate;
    p.epi.whole = p.N % 8 == 0 && aligned(out, 16) && ld_elements * es % 16 == 0;
}

// Operands whose rows begin on 16 bytes and hold whole 16-byte chunks are used where they lie, others through a padded copy
template <class T> struct Operands {
    CopyArgs C;
    Operands() { memset(&C, 0, sizeof(C)); }
    Matrix use(const void *src, size_t ld, size_t rows, size_t cols, Carve &w) {
        constexpr size_t es = sizeof(T);
        const size_t ld_dst = round_up(cols * es, 16);
        char *dst = w.take(rows * ld_dst);  // counted whether needed or not: the workspace's size does not depend on addresses
        if (aligned(src, 16) && ld % 16 == 0 && cols * es % 16 == 0) return Matrix{(const char *)src, ld};
        copy(src, ld, rows, cols, dst, ld_dst, 0);
        return Matrix{dst, ld_dst};
    }
    // two bf16 arrays whose sum the operand is, for run<true>()
    Matrix split(const void *src, size_t ld, size_t rows, size_t cols, size_t &apart, Carve &w) {
        const size_t ld_dst = round_up(cols * sizeof(T), 16);
        apart = round_up(rows * ld_dst, 256);
        char *dst = w.take(2 * apart);
        copy(src, ld, rows, cols, dst, ld_dst, apart);
        return Matrix{dst, ld_dst};
    }
    void copy(const void *src, size_t ld, size_t rows, size_t cols, char *dst, size_t ld_dst, size_t split) {
        CopyArgs::One &o = C.c[C.n++];
        o.src = (const char *)src; o.dst = dst; o.ld_src = ld; o.ld_dst = ld_dst; o.cols = (int)cols; o.chunks = (int)(ld_dst / 16); o.rows = rows; o.split = split;
    }
    template <bool SPLIT = false> void run(ckksmi_ctx *c, hipStream_t st) {
        // pieces of 256 chunks; several a workgroup where a launch would not hold as many workgroups
        size_t pieces = 0;
        for (int i = 0; i < C.n; i++) pieces += (C.c[i].rows * C.c[i].chunks + 255) / 256;
        C.per = (unsigned)(1 + pieces / TG_COPY_BLOCKS);
        unsigned blocks = 0;
        for (int i = 0; i < C.n; i++) {
            C.c[i].first = blocks;
            blocks += (unsigned)(((C.c[i].rows * C.c[i].chunks + 255) / 256 + C.per - 1) / C.per);
        }
        if (blocks) KL(c, CKKSMI_K_GEMM_COPY, blocks, (pad_rows_kernel<T, SPLIT>), dim3(blocks), dim3(256), st, C);
    }
};

// the products' shapes alone, for the workspace: as the passes below form them.  Never less for more rows: a workspace serves any number
// of rows up to the one it was made for (the weights' gradients have the rows for their k axis, and a longer one has no fewer parts)
size_t split_bytes(const ckksmi_gated_ff &f, bool backward) {
    const FF d(f);
    const Matrix none{nullptr, 0};
    auto one = [&](const GemmProblem &p, bool gate) { return part_bytes_up_to(p, gate, d.es) + 256; };
    size_t most = std::max(one(product(none, none, d.M, d.H, d.K), true), one(product(none, none, d.M, d.O, d.H), false));
    if (!backward || d.M == 0) return most;
    GemmProblem dx = product(none, none, d.M, d.K, d.H);
    dx.nsrc = 2;
    most = std::max(most, std::max(one(product(none, none, d.M, d.H, d.O), false), one(dx, false)));
    GemmProblem dw[3] = {product(none, none, d.H, d.K, d.M), product(none, none, d.H, d.K, d.M), product(none, none, d.O, d.H, d.M)};
    for (GemmProblem &p : dw) p.nsrc = d.sources(f.dtype);
    const int splits = choose(dw, 3, false, d.es).splits;
    return std::max(most, part_bytes(dw[0], splits, false) * 2 + part_bytes(dw[2], splits, false) + 768);
}

// Every product of the pass fits a launch: refused before anything is enqueued
int fits_grids(const ckksmi_gated_ff &f, bool backward) {
    const FF d(f);
    if (d.M == 0) return CKKSMI_OK;
    const Matrix none{nullptr, 0};
    auto fits = [&](const GemmProblem &p, bool gate) { return workgroups_of(&p, 1, gate, d.es) != 0; };
    bool ok = fits(product(none, none, d.M, d.H, d.K), true) && fits(product(none, none, d.M, d.O, d.H), false);
    if (ok && backward) {
        const GemmProblem dw[3] = {product(none, none, d.H, d.K, d.M), product(none, none, d.H, d.K, d.M), product(none, none, d.O, d.H, d.M)};
        ok = fits(product(none, none, d.M, d.H, d.O), false) && fits(product(none, none, d.M, d.K, d.H), false) && workgroups_of(dw, 3, false, d.es) != 0;
    }
    return ok ? CKKSMI_OK : CKKSMI_EUNSUPPORTED;
}

size_t workspace_of(const ckksmi_gated_ff &f, bool backward) {
    const FF d(f);
    auto rows = [&](size_t r, size_t cols) { return round_up(r * round_up(cols * d.es, 16), 256); };
    const size_t weights = 2 * rows(d.H, d.K) + rows(d.O, d.H);
    const size_t forward = rows(d.M, d.K) + weights + d.hidden_bytes();
    const size_t split = f.dtype == CKKSMI_F16 && d.fine() ? 2 * (rows(d.M, d.K) + rows(d.M, d.O)) : 0;
    const size_t back = rows(d.M, d.K) + weights + rows(d.M, d.O) + split + 2 * d.arrays(f.dtype) * d.hidden_bytes();
    return (backward ? std::max(forward, back) : forward) + split_bytes(f, backward);
}

// Few rows: products straight from the operands where they lie.  Up to 64 (64 f32 rows of 3136 -> 256: 22 us, by tiles in 24 parts and
// their join 29; one bf16 row of 1024 -> 4096 -> 1024: 14 us, by tiles 21)
constexpr int kFewRows = 64;
template <class T, int EPI>
void launch_rows(ckksmi_ctx *c, const RowsArgs &R, hipStream_t st) {
    const int blocks = (R.N + 15) / 16, tiles = (R.M + 15) / 16;
    const double flops = 2.0 * R.M * R.N * R.K * (EPI == EPI_GATE ? 2 : 1);
    // as many rows of x a workgroup as keep two workgroups a compute unit
    const int mt = blocks * tiles <= 512 ? 1 : blocks * ((tiles + 1) / 2) <= 512 ? 2 : 4;
    const dim3 grid(blocks, (tiles + mt - 1) / mt);
    switch (mt) {
        case 1: KL(c, CKKSMI_K_GEMM_ROWS, flops, (rows_kernel<T, EPI, 1, 16>), grid, dim3(1024), st, R); break;
        case 2: KL(c, CKKSMI_K_GEMM_ROWS, flops, (rows_kernel<T, EPI, 2, 8>), grid, dim3(512), st, R); break;
        default: KL(c, CKKSMI_K_GEMM_ROWS, flops, (rows_kernel<T, EPI, 4, 8>), grid, dim3(512), st, R); break;
    }
}

template <class T>
int forward(ckksmi_ctx *c, const ckksmi_gated_ff &f, const void *x, const void *wg, const void *wu, const void *wd, void *y, void *saved, Carve w, hipStream_t st) {
    const FF d(f);
    Guard guard(c);
    char *const keep = (char *)saved;
    EpiArgs to_hidden;
    memset(&to_hidden, 0, sizeof(to_hidden));
    if (keep) to_hidden.kept = d.kept(keep);
    to_hidden.arrays = keep ? d.arrays(f.dtype) : 1;
    to_hidden.array_bytes = d.hidden_bytes();
    to_hidden.ldo = d.ldh; to_hidden.N = (int)d.H; to_hidden.act = activation_of(f);
    if (d.M <= kFewRows) {
        RowsArgs R;
        memset(&R, 0, sizeof(R));
        char *const h = keep ? d.saved_h(keep) : w.take(d.hidden_bytes());
        R.x = (const char *)x; R.w[0] = (const char *)wg; R.w[1] = (const char *)wu; R.ldx = ld_bytes(f.ld_x, d.K, d.es); R.ldw = d.K * d.es;
        R.M = (int)d.M; R.N = (int)d.H; R.K = (int)d.K; R.epi = to_hidden; R.epi.o0 = h;
        launch_rows<T, EPI_GATE>(c, R, st);
        GemmProblem down = product(Matrix{h, d.ldh * d.es}, Matrix{(const char *)wd, d.H * d.es}, d.M, d.O, d.H);
        store_to(down, y, f.ld_y ? f.ld_y : d.O, f.dtype, false);
        R.x = h; R.w[0] = down.b[0]; R.ldx = down.lda; R.ldw = down.ldb;
        R.N = (int)d.O; R.K = (int)d.H; R.epi = down.epi;
        launch_rows<T, EPI_STORE>(c, R, st);
        return guard.rc();
    }
    Operands<T> ops;
    const Matrix mx = ops.use(x, ld_bytes(f.ld_x, d.K, d.es), d.M, d.K, w), mg = ops.use(wg, d.K * d.es, d.H, d.K, w), mu = ops.use(wu, d.K * d.es, d.H, d.K, w);
    const Matrix md = ops.use(wd, d.H * d.es, d.O, d.H, w);
    char *const h = keep ? d.saved_h(keep) : w.take(d.hidden_bytes());
    ops.run(c, st);

    GemmProblem gate = product(mx, mg, d.M, d.H, d.K);
    gate.b[1] = mu.p;
    gate.epi = to_hidden;
    gate.epi.o0 = h;
    launch_gemm<T, false, false, EPI_GATE>(c, &gate, 1, w, st);

    GemmProblem down = product(Matrix{h, d.ldh * d.es}, md, d.M, d.O, d.H);
    store_to(down, y, f.ld_y ? f.ld_y : d.O, f.dtype, false);
    launch_gemm<T, false, false, EPI_STORE>(c, &down, 1, w, st);
    return guard.rc();
}

template <class T>
int backward(ckksmi_ctx *c, const ckksmi_gated_ff &f, const void *x, const void *wg, const void *wu, const void *wd, const void *saved, const void *dy, void *dx,
             void *dwg, void *dwu, void *dwd, bool accumulate, Carve w, hipStream_t st) {
    const FF d(f);
    Guard guard(c);
    Operands<T> ops, halves;
    constexpr bool f16 = __is_same(T, _Float16);
    const size_t ldx = ld_bytes(f.ld_x, d.K, d.es), lddy = ld_bytes(f.ld_dy, d.O, d.es);
    const Matrix mg = ops.use(wg, d.K * d.es, d.H, d.K, w), mu = ops.use(wu, d.K * d.es, d.H, d.K, w), md = ops.use(wd, d.H * d.es, d.O, d.H, w);
    const Matrix mdy = ops.use(dy, lddy, d.M, d.O, w);
    // x and dy as the weights' gradients take them
    size_t x_apart = 0, dy_apart = 0;
    const bool split = f16 && d.fine();
    const Matrix gx = split ? halves.split(x, ldx, d.M, d.K, x_apart, w) : ops.use(x, ldx, d.M, d.K, w);
    const Matrix gdy = split ? halves.split(dy, lddy, d.M, d.O, dy_apart, w) : mdy;
    const int arrays = d.arrays(f.dtype);
    char *dg = w.take(arrays * d.hidden_bytes()), *du = w.take(arrays * d.hidden_bytes());
    const char *h = d.saved_h(saved);
    const size_t ldh = d.ldh * d.es;
    ops.run(c, st);
    if constexpr (f16) halves.template run<true>(c, st);

    GemmProblem dh = product(mdy, md, d.M, d.H, d.O);
    dh.epi.o0 = dg; dh.epi.o1 = du; dh.epi.arrays = arrays; dh.epi.array_bytes = d.hidden_bytes(); dh.epi.kept = d.kept(saved);
    dh.epi.ldo = d.ldh; dh.epi.N = (int)d.H;
    launch_gemm<T, false, true, EPI_DHID>(c, &dh, 1, w, st);

    if (dx) {
        GemmProblem p = product(Matrix{dg, ldh}, mg, d.M, d.K, d.H);
        p.a[1] = du; p.b[1] = mu.p; p.nsrc = 2;
        store_to(p, dx, f.ld_dx ? f.ld_dx : d.K, f.dtype, false);
        launch_gemm<T, false, true, EPI_STORE>(c, &p, 1, w, st);
    }
    GemmProblem dw[3] = {product(Matrix{dg, ldh}, gx, d.H, d.K, d.M), product(Matrix{du, ldh}, gx, d.H, d.K, d.M), product(gdy, Matrix{h, ldh}, d.O, d.H, d.M)};
    // arrays of h, dg, du and of x, dy whose products are added up (of f16 all but third part times second, 2^-24 of the whole)
    static const struct { int hidden, other; } bf16_sources[3] = {{0, 0}, {1, 0}, {2, 0}}, f16_sources[5] = {{1, 0}, {2, 0}, {1, 1}, {3, 0}, {2, 1}};
    for (GemmProblem &p : dw) p.nsrc = d.sources(f.dtype);
    for (int i = 0; d.fine() && i < dw[0].nsrc; i++) {
        const size_t at = (f16 ? f16_sources[i] : bf16_sources[i]).hidden * d.hidden_bytes(), other = (f16 ? f16_sources[i] : bf16_sources[i]).other;
        dw[0].a[i] = dg + at; dw[1].a[i] = du + at; dw[2].b[i] = h + at;
        dw[0].b[i] = dw[1].b[i] = gx.p + other * x_apart;
        dw[2].a[i] = gdy.p + other * dy_apart;
    }
    store_to(dw[0], dwg, d.K, f.grad_dtype, accumulate);
    store_to(dw[1], dwu, d.K, f.grad_dtype, accumulate);
    store_to(dw[2], dwd, d.H, f.grad_dtype, accumulate);
    if (split) launch_gemm<__bf16, true, true, EPI_STORE>(c, dw, 3, w, st);
    else launch_gemm<T, true, true, EPI_STORE>(c, dw, 3, w, st);
    return guard.rc();
}

// gradients of no rows
__global__ void __launch_bounds__(256) clear_kernel(char *p, size_t bytes) {
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < bytes; i += (size_t)gridDim.x * 256) p[i] = 0;
}

}  // namespace

extern "C" int ckksmi_gated_ff_workspace_bytes(const ckksmi_ctx *c, const ckksmi_gated_ff *ff, int backward, size_t *bytes) {
    if (!c || !ff || !bytes) return CKKSMI_EINVAL;
    const ckksmi_gated_ff f = *ff;
    int rc = check_ff(f);
    if (!rc) rc = fits_grids(f, backward != 0);
    if (rc) return rc;
    *bytes = workspace_of(f, backward != 0);
    return CKKSMI_OK;
}

extern "C" int ckksmi_gated_ff_saved_bytes(const ckksmi_ctx *c, const ckksmi_gated_ff *ff, size_t *bytes) {
    if (!c || !ff || !bytes) return CKKSMI_EINVAL;
    const ckksmi_gated_ff f = *ff;
    int rc = check_ff(f);
    if (!rc) rc = fits_grids(f, false);
    if (rc) return rc;
    *bytes = FF(f).saved_bytes(f.dtype);
    return CKKSMI_OK;
}

extern "C" int ckksmi_gated_ff_forward(ckksmi_ctx *c, const ckksmi_gated_ff *ff, const void *x, const void *wg, const void *wu, const void *wd, void *y, void *saved,
                                       void *ws, size_t ws_bytes, void *stream) {
    if (!dev_ok(c)) return CKKSMI_EDEVICE;
    if (!ff) return CKKSMI_EINVAL;
    const ckksmi_gated_ff f = *ff;
    int rc = check_ff(f);
    if (!rc) rc = fits_grids(f, false);
    if (rc) return rc;
    if (!wg || !wu || !wd) return CKKSMI_EINVAL;
    if (f.rows == 0) return CKKSMI_OK;
    const FF d(f);
    if (!x || !y || !ws || !aligned(ws, 16) || !aligned(saved, 16)) return CKKSMI_EINVAL;
    for (const void *p : {x, wg, wu, wd, (const void *)y})
        if (!aligned(p, d.es)) return CKKSMI_EINVAL;
    const size_t ldx = ld_bytes(f.ld_x, d.K, d.es), ldy = ld_bytes(f.ld_y, d.O, d.es);
    const size_t nx = (d.M - 1) * ldx + d.K * d.es, ny = (d.M - 1) * ldy + d.O * d.es, nw = d.H * d.K * d.es, nd = d.O * d.H * d.es, ns = saved ? d.saved_bytes(f.dtype) : 0;
    const void *in[4] = {x, wg, wu, wd};
    const size_t n_in[4] = {nx, nw, nw, nd};
    const size_t need = workspace_of(f, false);
    for (int i = 0; i < 4; i++)
        if (overlap(y, ny, in[i], n_in[i]) || overlap(saved, ns, in[i], n_in[i]) || overlap(ws, need, in[i], n_in[i])) return CKKSMI_EINVAL;
    if (overlap(y, ny, saved, ns) || overlap(ws, need, y, ny) || overlap(ws, need, saved, ns)) return CKKSMI_EINVAL;
    if (ws_bytes < need) return CKKSMI_EWORKSPACE;
    const Carve w(ws);
    switch (f.dtype) {
        case CKKSMI_F32: return forward<float>(c, f, x, wg, wu, wd, y, saved, w, S(stream));
        case CKKSMI_BF16: return forward<__bf16>(c, f, x, wg, wu, wd, y, saved, w, S(stream));
        default: return forward<_Float16>(c, f, x, wg, wu, wd, y, saved, w, S(stream));
    }
}

extern "C" int ckksmi_gated_ff_backward(ckksmi_ctx *c, const ckksmi_gated_ff *ff, const void *x, const void *wg, const void *wu, const void *wd, const void *saved,
                                        const void *dy, void *dx, void *dwg, void *dwu, void *dwd, int accumulate, void *ws, size_t ws_bytes, void *stream) {
    if (!dev_ok(c)) return CKKSMI_EDEVICE;
    if (!ff) return CKKSMI_EINVAL;
    const ckksmi_gated_ff f = *ff;
    int rc = check_ff(f);
    if (!rc) rc = fits_grids(f, true);
    if (rc) return rc;
    const FF d(f);
    if (!wg || !wu || !wd || !dwg || !dwu || !dwd) return CKKSMI_EINVAL;
    for (const void *p : {(const void *)dwg, (const void *)dwu, (const void *)dwd})
        if (!aligned(p, d.ges)) return CKKSMI_EINVAL;
    const size_t gw = d.H * d.K * d.ges, gd = d.O * d.H * d.ges;
    if (overlap(dwg, gw, dwu, gw) || overlap(dwg, gw, dwd, gd) || overlap(dwu, gw, dwd, gd)) return CKKSMI_EINVAL;
    if (f.rows == 0) {  // sums of nothing
        if (accumulate) return CKKSMI_OK;
        Guard guard(c);
        KL(c, CKKSMI_K_GEMM_COPY, 1, clear_kernel, dim3(1024), dim3(256), S(stream), (char *)dwg, gw);
        KL(c, CKKSMI_K_GEMM_COPY, 1, clear_kernel, dim3(1024), dim3(256), S(stream), (char *)dwu, gw);
        KL(c, CKKSMI_K_GEMM_COPY, 1, clear_kernel, dim3(1024), dim3(256), S(stream), (char *)dwd, gd);
        return guard.rc();
    }
    if (!x || !dy || !saved || !ws || !aligned(ws, 16) || !aligned(saved, 16)) return CKKSMI_EINVAL;
    for (const void *p : {x, wg, wu, wd, dy, (const void *)dx})
        if (!aligned(p, d.es)) return CKKSMI_EINVAL;
    const size_t nw = d.H * d.K * d.es, nd = d.O * d.H * d.es;
    auto span = [&](int64_t ld, size_t cols) { return (d.M - 1) * ld_bytes(ld, cols, d.es) + cols * d.es; };
    const size_t need = workspace_of(f, true);
    const void *in[6] = {x, wg, wu, wd, saved, dy};
    const size_t n_in[6] = {span(f.ld_x, d.K), nw, nw, nd, d.saved_bytes(f.dtype), span(f.ld_dy, d.O)};
    const void *out[4] = {dx, dwg, dwu, dwd};
    const size_t n_out[4] = {dx ? span(f.ld_dx, d.K) : 0, gw, gw, gd};
    for (int o = 0; o < 4; o++) {
        for (int i = 0; i < 6; i++)
            if (overlap(out[o], n_out[o], in[i], n_in[i])) return CKKSMI_EINVAL;
        if (overlap(out[o], n_out[o], ws, need) || (o && overlap(out[0], n_out[0], out[o], n_out[o]))) return CKKSMI_EINVAL;
    }
    for (int i = 0; i < 6; i++)
        if (overlap(ws, need, in[i], n_in[i])) return CKKSMI_EINVAL;
    if (ws_bytes < need) return CKKSMI_EWORKSPACE;
    const Carve w(ws);
    switch (f.dtype) {
        case CKKSMI_F32: return backward<float>(c, f, x, wg, wu, wd, saved, dy, dx, dwg, dwu, dwd, accumulate != 0, w, S(stream));
        case CKKSMI_BF16: return backward<__bf16>(c, f, x, wg, wu, wd, saved, dy, dx, dwg, dwu, dwd, accumulate != 0, w, S(stream));
        default: return backward<_Float16>(c, f, x, wg, wu, wd, saved, dy, dx, dwg, dwu, dwd, accumulate != 0, w, S(stream));
    }
}

// ------------------------------------------------------------------ AdamW
static int check_tensor(const ckksmi_adamw_tensor &t, size_t p_align, size_t g_align, size_t copy_align, bool bytes) {
    if (t.n < 0 || t.n > kMaxNumel) return CKKSMI_EINVAL;
    if (t.n == 0) return CKKSMI_OK;
    if (!t.p || !t.grad || !t.m || !t.v || !aligned(t.p, p_align) || !aligned(t.grad, g_align) || !aligned(t.copy, copy_align)) return CKKSMI_EINVAL;
    if (bytes) return t.m_unit && t.v_unit && aligned(t.m_unit, 4) && aligned(t.v_unit, 4) ? CKKSMI_OK : CKKSMI_EINVAL;
    return aligned(t.m, 4) && aligned(t.v, 4) ? CKKSMI_OK : CKKSMI_EINVAL;
}

template <class P, int BITS>
static void launch_adamw(ckksmi_ctx *c, const AdamwArgs &A, int grad_dtype, unsigned blocks, hipStream_t st) {
    const double units = (double)blocks * TA_CHUNK;
    switch (grad_dtype) {
        case CKKSMI_F32: KL(c, CKKSMI_K_ADAMW, units, (adamw_kernel<P, float, BITS>), dim3(blocks), dim3(256), st, A); break;
        case CKKSMI_BF16: KL(c, CKKSMI_K_ADAMW, units, (adamw_kernel<P, __bf16, BITS>), dim3(blocks), dim3(256), st, A); break;
        default: KL(c, CKKSMI_K_ADAMW, units, (adamw_kernel<P, _Float16, BITS>), dim3(blocks), dim3(256), st, A); break;
    }
}

extern "C" int ckksmi_adamw_step(ckksmi_ctx *c, const ckksmi_adamw *opt, const ckksmi_adamw_tensor *t, int n_tensors, void *stream) {
    if (!dev_ok(c)) return CKKSMI_EDEVICE;
    if (!opt) return CKKSMI_EINVAL;
    const ckksmi_adamw o = *opt;
    if (n_tensors < 0 || (!t && n_tensors) || !dtype_ok(o.p_dtype) || !dtype_ok(o.grad_dtype) || (o.state_bits != 8 && o.state_bits != 32)) return CKKSMI_EINVAL;
    if (o.step < 1 || !(o.beta1 >= 0 && o.beta1 < 1) || !(o.beta2 >= 0 && o.beta2 < 1) || !(o.eps >= 0) || !std::isfinite(o.eps) || !std::isfinite(o.lr) ||
        !std::isfinite(o.weight_decay) || !std::isfinite(o.grad_scale) || !aligned(o.skip, 4))
        return CKKSMI_EINVAL;
    bool copies = false;
    for (int i = 0; i < n_tensors; i++) copies = copies || (t[i].n > 0 && t[i].copy);
    if (copies && o.copy_dtype != CKKSMI_BF16 && o.copy_dtype != CKKSMI_F16) return CKKSMI_EINVAL;
    const bool bytes = o.state_bits == 8;
    for (int i = 0; i < n_tensors; i++) {
        const int rc = check_tensor(t[i], element_bytes(o.p_dtype), element_bytes(o.grad_dtype), 2, bytes);
        if (rc) return rc;
    }
    AdamwArgs A;
    memset(&A, 0, sizeof(A));
    A.copy_f16 = o.copy_dtype == CKKSMI_F16;
    A.key = adamw_mix(adamw_mix((unsigned)o.seed) + (unsigned)(o.seed >> 32));
    A.beta1 = (float)o.beta1; A.rest1 = (float)(1.0 - o.beta1);
    A.beta2 = (float)o.beta2; A.rest2 = (float)(1.0 - o.beta2);
    A.decay = (float)(1.0 - o.lr * o.weight_decay);
    A.size = (float)(o.lr / (1.0 - std::pow(o.beta1, (double)o.step)));
    A.root = (float)(1.0 / std::sqrt(1.0 - std::pow(o.beta2, (double)o.step)));
    A.eps = (float)o.eps; A.grad_scale = (float)o.grad_scale; A.skip = o.skip;
    Guard guard(c);
    for (int i = 0; i < n_tensors;) {
        // as many tensors as the table holds and a grid may have workgroups (one tensor's always fit: kMaxNumel)
        size_t blocks = 0;
        A.tensor0 = i;
        A.n = 0;
        while (i < n_tensors && A.n < TA_TENSORS) {
            const size_t more = (size_t)(t[i].n + TA_CHUNK - 1) / TA_CHUNK;
            if (blocks + more > kMaxBlocks) break;
            A.t[A.n] = t[i];
            A.first[A.n++] = (unsigned)blocks;
            blocks += more;
            i++;
        }
        A.first[A.n] = (unsigned)blocks;
        if (blocks == 0) continue;
        switch (o.p_dtype * 64 + o.state_bits) {
            case CKKSMI_F32 * 64 + 32: launch_adamw<float, 32>(c, A, o.grad_dtype, (unsigned)blocks, S(stream)); break;
            case CKKSMI_F32 * 64 + 8: launch_adamw<float, 8>(c, A, o.grad_dtype, (unsigned)blocks, S(stream)); break;
            case CKKSMI_BF16 * 64 + 32: launch_adamw<__bf16, 32>(c, A, o.grad_dtype, (unsigned)blocks, S(stream)); break;
            case CKKSMI_BF16 * 64 + 8: launch_adamw<__bf16, 8>(c, A, o.grad_dtype, (unsigned)blocks, S(stream)); break;
            case CKKSMI_F16 * 64 + 32: launch_adamw<_Float16, 32>(c, A, o.grad_dtype, (unsigned)blocks, S(stream)); break;
            default: launch_adamw<_Float16, 8>(c, A, o.grad_dtype, (unsigned)blocks, S(stream)); break;
        }
    }
    return guard.rc();
}

extern "C" int ckksmi_adamw_read_states(ckksmi_ctx *c, const ckksmi_adamw_tensor *t, int n_tensors, float *const *m_out, float *const *v_out, void *stream) {
    if (!dev_ok(c)) return CKKSMI_EDEVICE;
    if (n_tensors < 0 || (!t && n_tensors) || (!m_out && !v_out)) return CKKSMI_EINVAL;
    for (int i = 0; i < n_tensors; i++) {
        if (t[i].n < 0 || t[i].n > kMaxNumel) return CKKSMI_EINVAL;
        if (t[i].n == 0) continue;
        if (m_out && (!m_out[i] || !t[i].m || !t[i].m_unit || !aligned(m_out[i], 4) || !aligned(t[i].m_unit, 4))) return CKKSMI_EINVAL;
        if (v_out && (!v_out[i] || !t[i].v || !t[i].v_unit || !aligned(v_out[i], 4) || !aligned(t[i].v_unit, 4))) return CKKSMI_EINVAL;
    }
    ReadStatesArgs A;
    memset(&A, 0, sizeof(A));
    Guard guard(c);
    for (int i = 0; i < n_tensors;) {
        size_t blocks = 0;
        A.n = 0;
        while (i < n_tensors && A.n < TA_TENSORS) {
            const size_t more = (size_t)(t[i].n + TA_CHUNK - 1) / TA_CHUNK;
            if (blocks + more > kMaxBlocks) break;
            ReadStatesArgs::One &o = A.t[A.n];
            o.m = (const unsigned char *)t[i].m; o.v = (const unsigned char *)t[i].v; o.m_unit = t[i].m_unit; o.v_unit = t[i].v_unit;
            o.m_out = m_out ? m_out[i] : nullptr; o.v_out = v_out ? v_out[i] : nullptr; o.n = t[i].n;
            A.first[A.n++] = (unsigned)blocks;
            blocks += more;
            i++;
        }
        if (blocks) KL(c, CKKSMI_K_ADAMW_READ, (double)blocks * TA_CHUNK, adamw_read_kernel, dim3((unsigned)blocks), dim3(256), S(stream), A);
    }
    return guard.rc();
}
