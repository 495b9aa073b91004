// Orthogonalised directions and steps along them (include/ckksmi_train.h): argument checks, workspaces and launch sequences.
#include "train_call.h"
#include "train_series.h"

namespace {

constexpr int64_t kMaxSide = 1 << 16;
#ifndef TG_ENOUGH_TILES
#define TG_ENOUGH_TILES 192  // three quarters of the compute units (the tests' stand-in sets it)
#endif

#ifndef TS_SMALL_MOST
#define TS_SMALL_MOST TS_SMALL_LDS  // bytes of LDS up to which a call's matrices take one workgroup each (the tests' stand-in sets it)
#endif

#ifndef TS_TILE
#define TS_TILE(rule) (rule)  // which of the large tiles (the tests' stand-in may choose)
#endif

// The polynomials keep singular values and entries where f16 holds them: the largest value that can stand at each step's end, on a grid
// fine enough for a polynomial of degree five.  of_b: the power of two that takes the entries of b A + c A^2 near f16's end
int check_series(const ckksmi_series &s, float *of_b = nullptr) {
    double entries = 1.0;
    if (s.steps < 1 || s.steps > 32 || !(s.eps >= 0) || !std::isfinite(s.eps) || !std::isfinite(s.a) || !std::isfinite(s.b) || !std::isfinite(s.c)) return CKKSMI_EINVAL;
    double most = 1.0;
    for (int k = 0; k < s.steps; k++) {
        const double entry = std::fabs(s.b) * most * most + std::fabs(s.c) * most * most * most * most;
        if (!(entry < 100.0)) return CKKSMI_EINVAL;
        entries = std::max(entries, entry);
        double next = 0.0;
        for (int i = 0; i <= 1024; i++) {
            const double v = most * i / 1024.0, w = v * v;
            next = std::max(next, std::fabs(v * (s.a + w * (s.b + w * s.c))));
        }
        if (!(next < 2.0)) return CKKSMI_EINVAL;
        most = std::max(most, next);
    }
    if (of_b) *of_b = (float)std::ldexp(1.0, (int)std::floor(std::log2(52000.0 / entries)));
    return CKKSMI_OK;
}

// What both entry points make of their tensors
struct SeriesTensor {
    void *p, *copy;
    const void *g;
    float *m;
    int64_t rows, cols;
    double scale;
};

// A tensor's sizes and its pieces of the workspace
struct SeriesPlan {
    int side, length, ld, ld_o, blocks;
    size_t numel, per;
    explicit SeriesPlan(const SeriesTensor &t) {
        side = (int)std::min(t.rows, t.cols);
        length = (int)std::max(t.rows, t.cols);
        ld = (int)round_up(length, 8);
        ld_o = (int)round_up(side, 8);
        numel = (size_t)t.rows * t.cols;
        // the first pass: at most 1024 workgroups' sums, which every workgroup of the second adds up
        per = round_up((numel + 1023) / 1024, 4096);
        blocks = (int)((numel + per - 1) / per);
    }
    // everything in one workgroup's LDS
    bool small() const { return side <= 64 && small_lds(side, length) <= TS_SMALL_MOST; }
    size_t x_bytes() const { return (size_t)side * ld * 4; }  // two parts of f16, or a direction in f32
    size_t o_bytes() const { return (size_t)side * ld_o * 4; }  // two parts
    // X and its successor, O, B, two diagonals, sums of squares
    size_t bytes() const {
        return 2 * round_up(x_bytes(), 256) + 2 * round_up(o_bytes(), 256) + 2 * round_up((size_t)side * 4, 256) + round_up((size_t)blocks * 8, 256);
    }
};
struct SeriesPieces { char *x[2], *o, *b; float *d, *e; double *sums; };

struct SeriesShape { int bm, bn; };
constexpr SeriesShape kSeriesTiles[3] = {{256, 256}, {128, 128}, {32, 128}};
struct SeriesLaunch { int tile, splits; };

long long series_tiles(const SeriesProblem &p, const SeriesShape &t, bool triangle, SeriesProblem *out) {
    const int tm = (p.M + t.bm - 1) / t.bm, tn = (p.N + t.bn - 1) / t.bn;
    if (out) { out->tiles_m = tm; out->tiles_n = tn; }
    if (!triangle) return (long long)tm * tn;
    const long long R = t.bn / t.bm, whole = tm / R, rest = tm % R;  // groups of R tile rows have one tile more each
    return R * (whole * (whole + 1) / 2) + rest * (whole + 1);
}
inline int series_steps(const SeriesProblem &p) { return (p.K + 63) / 64 * p.nsrc; }

// Tile and parts of the k axis of a launch.  Measured, us of a whole direction (three products of each kind):
//   enough 128 x 128 tiles for three quarters of the compute units: those or 256 x 256, by rounds of the compute units, which hold one of 256 or two of 128
//       (a round of the smaller takes 0.72 of the larger's; all in tiles of 256, 128: one 4096 x 4096 4340, 5290; 8192 x 8192, 528 tiles of 256 or 2080
//       of 128 for the symmetric products, 32400, 39300, and with 128 there alone 36000; 6144 x 6144 15730, 16190; twelve of 1024 x 4096,
//       whose X X^T has 120 or 432: 3800, 3530, and with 256 for X's product alone 3270)
//   enough 32 x 128 tiles: those, the k axis whole (2048 x 2048, 544: 1080, 136 of 128 1200)
//   few tiles and a long k axis: 128 x 128 in parts (X X^T of 1024 x 4096: 8 parts 599, 4 632, 32 x 128 whole 667, in 4 parts 612)
//   else 32 x 128, with four groups of waves for a tile's k axis (launch_series); in parts where that leaves half of the compute units idle
//       (the square and X X^T of 1024 x 1024: 32 x 128 whole 377, two parts 428, 128 x 128 in 4 421; X X^T of two 256 x 3136: 8 parts 212, 4 231, whole 336)
SeriesLaunch series_choose(const SeriesProblem *p, int n, bool triangle) {
    long long tiles[3] = {0, 0, 0};
    int steps = 0;
    for (int i = 0; i < n; i++) {
        for (int t = 0; t < 3; t++) tiles[t] += series_tiles(p[i], kSeriesTiles[t], triangle, nullptr);
        steps = std::max(steps, series_steps(p[i]));
    }
    const long long units = 4 * TG_ENOUGH_TILES / 3;  // compute units
    auto rounds = [](long long tiles, long long held) { return (double)((tiles + held - 1) / held); };
    auto parts = [&](int t) { return (int)std::max(1LL, std::min(std::min(256 / tiles[t], (long long)steps / 16), 32LL)); };
    if (tiles[1] >= TG_ENOUGH_TILES) return SeriesLaunch{TS_TILE(rounds(tiles[0], units) <= 0.72 * rounds(tiles[1], 2 * units) ? 0 : 1), 1};
    if (tiles[2] >= 256) return SeriesLaunch{2, 1};
    if (steps >= 128 && tiles[1] >= 24) return SeriesLaunch{1, parts(1)};
    return SeriesLaunch{2, parts(2)};
}
inline size_t series_part_bytes(const SeriesProblem &p, int splits) { return splits > 1 ? round_up((size_t)splits * p.M * round_up(p.N, 8) * sizeof(float), 256) : 0; }

template <int EPI> void launch_series(ckksmi_ctx *c, SeriesProblem *p, int n, char *part, hipStream_t st) {
    constexpr bool triangle = symmetric(EPI), b_rows = EPI == EPI_APPLY;
    const SeriesLaunch s = series_choose(p, n, triangle);
    SeriesArgs G;
    memset(&G, 0, sizeof(G));
    int total = 0, join = 0, steps = 0;
    double flops = 0;
    for (int i = 0; i < n; i++) {
        G.first[i] = total;
        total += (int)series_tiles(p[i], kSeriesTiles[s.tile], triangle, &p[i]);
        p[i].ld_part = round_up(p[i].N, 8);
        p[i].part = (float *)part;
        part += series_part_bytes(p[i], s.splits);
        G.p[i] = p[i];
        join = std::max(join, (int)(((size_t)p[i].M * p[i].ld_part / 8 + 255) / 256));
        steps = std::max(steps, series_steps(p[i]));
        flops += 2.0 * p[i].M * p[i].N * p[i].K * p[i].nsrc * (triangle ? 0.5 : 1.0);
    }
    G.first[n] = total;
    G.n_problems = n;
    G.splits = s.splits;
    const dim3 grid(total, s.splits);
    if (s.tile == 0) KL(c, CKKSMI_K_SERIES, flops, (gemm_kernel<_Float16, 256, 256, 128, 64, false, b_rows, EPI, SeriesArgs>), grid, dim3(512), st, G);
    if (s.tile == 1) KL(c, CKKSMI_K_SERIES, flops, (gemm_kernel<_Float16, 128, 128, 64, 64, false, b_rows, EPI, SeriesArgs>), grid, dim3(256), st, G);
    const bool groups = s.tile == 2 && total * s.splits <= 256 && steps > 2 * s.splits;
    if (groups) KL(c, CKKSMI_K_SERIES, flops, (gemm_small_kernel<_Float16, 32, 128, 16, 64, 4, false, b_rows, EPI, SeriesArgs>), grid, dim3(1024), st, G);
    else if (s.tile == 2) KL(c, CKKSMI_K_SERIES, flops, (gemm_small_kernel<_Float16, 32, 128, 16, 64, 1, false, b_rows, EPI, SeriesArgs>), grid, dim3(256), st, G);
    if (s.splits > 1) KL(c, CKKSMI_K_SERIES_JOIN, flops, (series_join_kernel<EPI>), dim3(join, n), dim3(256), st, G);
}

// A tensor's products of a step; pieces null: their sizes alone
SeriesProblem series_problem(const SeriesPlan &t, const SeriesPieces &w, const ckksmi_series &s, float of_b, int epi, int from, bool last) {
    SeriesProblem p;
    memset(&p, 0, sizeof(p));
    const size_t x_part = (size_t)t.side * t.ld * 2, o_part = (size_t)t.side * t.ld_o * 2;
    const char *a = epi == EPI_GRAM ? w.x[from] : epi == EPI_SQUARE ? w.o : w.b, *b = epi == EPI_SQUARE ? w.o : w.x[from];
    const size_t a_part = epi == EPI_GRAM ? x_part : o_part, b_part = epi == EPI_SQUARE ? o_part : x_part;
    p.nsrc = 3;
    for (int i = 0; i < 3; i++) {  // upper times lower, lower times upper, upper times upper
        p.a[i] = a + (i == 1 ? a_part : 0);
        p.b[i] = b + (i == 0 ? b_part : 0);
    }
    p.lda = (epi == EPI_GRAM ? t.ld : t.ld_o) * 2;
    p.ldb = (epi == EPI_SQUARE ? t.ld_o : t.ld) * 2;
    p.M = t.side;
    p.N = epi == EPI_APPLY ? t.length : t.side;
    p.K = epi == EPI_GRAM ? t.length : t.side;
    p.ca = (float)s.a; p.cb = (float)s.b; p.cc = (float)s.c; p.of_b = of_b;
    p.apart = (epi == EPI_APPLY ? x_part : o_part) / 2;
    p.ldo = epi == EPI_APPLY ? t.ld : t.ld_o;
    if (epi == EPI_GRAM) {
        p.o = (_Float16 *)w.o; p.diag_out = w.d;
    } else if (epi == EPI_SQUARE) {
        p.o = (_Float16 *)w.b; p.in = (const _Float16 *)w.o; p.diag = w.d; p.diag_out = w.e;
    } else {
        p.in = (const _Float16 *)w.x[from]; p.diag = w.e;
        if (last) p.last = (float *)w.x[1 - from];
        else p.o = (_Float16 *)w.x[1 - from];
    }
    return p;
}

// Workspace of a call: its tensors' pieces and the largest of what launches need for k axes in parts
size_t series_workspace(const std::vector<SeriesPlan> &plans, const ckksmi_series &s) {
    size_t total = 0, most = 0;
    const SeriesPieces none{};
    for (const SeriesPlan &t : plans) total += t.bytes();
    for (size_t i = 0; i < plans.size(); i += TS_PROBLEMS) {
        const int n = (int)std::min<size_t>(TS_PROBLEMS, plans.size() - i);
        for (int epi : {EPI_GRAM, EPI_SQUARE, EPI_APPLY}) {
            SeriesProblem p[TS_PROBLEMS];
            for (int k = 0; k < n; k++) p[k] = series_problem(plans[i + k], none, s, 1.0f, epi, 0, false);
            const int splits = series_choose(p, n, symmetric(epi)).splits;
            size_t need = 0;
            for (int k = 0; k < n; k++) need += series_part_bytes(p[k], splits);
            most = std::max(most, need);
        }
    }
    return total + most;
}

// (vectors' memory may not be there: the entry points turn that into an error)
struct SeriesCall {
    std::vector<SeriesTensor> t;
    std::vector<SeriesPlan> plan;
    size_t need;
    float of_b = 1.0f;
    bool small = true;  // all of them are
    SeriesCall(std::vector<SeriesTensor> tensors, const ckksmi_series &s) {
        (void)check_series(s, &of_b);  // (it has passed)
        for (const SeriesTensor &x : tensors)
            if (x.rows && x.cols) {
                t.push_back(x);
                plan.emplace_back(x);
                small = small && plan.back().small();
            }
        need = small ? 0 : series_workspace(plan, s);
    }
};

// One of the passes over all tensors' elements, in as few launches as their tables allow.  blocks_of: a tensor's workgroups
template <class Blocks, class Launch> void for_tables(const SeriesCall &call, const std::vector<SeriesPieces> &w, PassArgs A, int direction, Blocks blocks_of, Launch launch) {
    for (size_t i = 0; i < call.t.size();) {
        int64_t blocks = 0;
        A.n = 0;
        while (i < call.t.size() && A.n < TS_TENSORS) {
            const int64_t more = blocks_of(call.plan[i]);
            if (A.n && blocks + more > kMaxBlocks) break;
            const SeriesTensor &s = call.t[i];
            const SeriesPlan &l = call.plan[i];
            PassTensor &t = A.t[A.n];
            t.p = (char *)s.p; t.g = (const char *)s.g; t.m = s.m; t.copy = (char *)s.copy;
            if (!call.small) {
                t.sums = w[i].sums; t.x = (_Float16 *)w[i].x[0]; t.o = (_Float16 *)w[i].o; t.b = (_Float16 *)w[i].b; t.direction = (const float *)w[i].x[direction];
            }
            t.numel = (int64_t)l.numel; t.per = (int64_t)l.per; t.rows = (int)s.rows; t.cols = (int)s.cols; t.ld = l.ld; t.ld_o = l.ld_o;
            t.scale = (float)s.scale; t.blocks = l.blocks;
            A.first[A.n++] = (unsigned)blocks;
            blocks += more;
            i++;
        }
        A.first[A.n] = (unsigned)blocks;
        launch(A, (unsigned)blocks);
    }
}
inline int64_t series_squares(const SeriesPlan &l) { return (int64_t)((l.side + 63) / 64) * ((l.ld + 63) / 64); }

template <class P, class G, bool MOVE> void run_small(ckksmi_ctx *c, const SeriesCall &call, const ckksmi_series &s, const PassArgs &A, hipStream_t st) {
    const SmallSeries S{s.steps, (float)s.a, (float)s.b, (float)s.c, call.of_b};
    for_tables(call, {}, A, 0, [](const SeriesPlan &) { return (int64_t)1; }, [&](const PassArgs &a, unsigned blocks) {
        double flops = 0;  // three products of each kind, half of the symmetric ones
        for (int i = 0; i < a.n; i++) {
            const double m = std::min(a.t[i].rows, a.t[i].cols), n = std::max(a.t[i].rows, a.t[i].cols);
            flops += 3.0 * s.steps * (m * m * n + m * m * m + 2.0 * m * m * n);
        }
        KL(c, CKKSMI_K_SERIES_SMALL, flops, (series_small_kernel<P, G, MOVE>), dim3(blocks), dim3(TS_SMALL_THREADS), st, a, S);
    });
}
template <class P, bool MOVE> void run_series(ckksmi_ctx *c, const SeriesCall &call, const ckksmi_series &s, const PassArgs &A, void *ws, hipStream_t st) {
    if (call.small) {
        switch (A.g_dtype) {
            case CKKSMI_F32: run_small<P, float, MOVE>(c, call, s, A, st); break;
            case CKKSMI_BF16: run_small<P, __bf16, MOVE>(c, call, s, A, st); break;
            default: run_small<P, _Float16, MOVE>(c, call, s, A, st); break;
        }
        return;
    }
    Carve carve(ws);
    std::vector<SeriesPieces> w;
    for (const SeriesPlan &l : call.plan) {
        SeriesPieces p;
        p.x[0] = carve.take(l.x_bytes()); p.x[1] = carve.take(l.x_bytes());
        p.o = carve.take(l.o_bytes()); p.b = carve.take(l.o_bytes());
        p.d = (float *)carve.take((size_t)l.side * 4); p.e = (float *)carve.take((size_t)l.side * 4);
        p.sums = (double *)carve.take((size_t)l.blocks * 8);
        w.push_back(p);
    }
    char *const part = (char *)ws + carve.used;
    for_tables(call, w, A, 0, [](const SeriesPlan &l) { return (int64_t)l.blocks; }, [&](const PassArgs &a, unsigned blocks) {
        switch (A.g_dtype) {
            case CKKSMI_F32: KL(c, CKKSMI_K_SERIES_PASS, blocks, (series_momentum_kernel<float>), dim3(blocks), dim3(256), st, a); break;
            case CKKSMI_BF16: KL(c, CKKSMI_K_SERIES_PASS, blocks, (series_momentum_kernel<__bf16>), dim3(blocks), dim3(256), st, a); break;
            default: KL(c, CKKSMI_K_SERIES_PASS, blocks, (series_momentum_kernel<_Float16>), dim3(blocks), dim3(256), st, a); break;
        }
    });
    for_tables(call, w, A, 0, series_squares, [&](const PassArgs &a, unsigned blocks) {
        switch (A.g_dtype) {
            case CKKSMI_F32: KL(c, CKKSMI_K_SERIES_PASS, blocks, (series_begin_kernel<float>), dim3(blocks), dim3(256), st, a); break;
            case CKKSMI_BF16: KL(c, CKKSMI_K_SERIES_PASS, blocks, (series_begin_kernel<__bf16>), dim3(blocks), dim3(256), st, a); break;
            default: KL(c, CKKSMI_K_SERIES_PASS, blocks, (series_begin_kernel<_Float16>), dim3(blocks), dim3(256), st, a); break;
        }
    });
    for (int k = 0; k < s.steps; k++)
        for (size_t i = 0; i < w.size(); i += TS_PROBLEMS) {
            const int n = (int)std::min<size_t>(TS_PROBLEMS, w.size() - i);
            SeriesProblem p[TS_PROBLEMS];
            auto all = [&](int epi) {
                for (int j = 0; j < n; j++) p[j] = series_problem(call.plan[i + j], w[i + j], s, call.of_b, epi, k & 1, k + 1 == s.steps);
            };
            all(EPI_GRAM);
            launch_series<EPI_GRAM>(c, p, n, part, st);
            all(EPI_SQUARE);
            launch_series<EPI_SQUARE>(c, p, n, part, st);
            all(EPI_APPLY);
            launch_series<EPI_APPLY>(c, p, n, part, st);
        }
    for_tables(call, w, A, s.steps & 1, series_squares, [&](const PassArgs &a, unsigned blocks) {
        KL(c, CKKSMI_K_SERIES_PASS, blocks, (series_end_kernel<P, MOVE>), dim3(blocks), dim3(256), st, a);
    });
}

int check_sizes(int64_t rows, int64_t cols) { return rows < 0 || cols < 0 || rows > kMaxSide || cols > kMaxSide ? CKKSMI_EINVAL : CKKSMI_OK; }

int directions_call(const ckksmi_series *s, const ckksmi_direction *t, int n, int dtype, ckksmi_series &series, std::vector<SeriesTensor> &out) {
    if (!s || n < 0 || (!t && n) || !dtype_ok(dtype)) return CKKSMI_EINVAL;
    series = *s;
    const int rc = check_series(series);
    if (rc) return rc;
    for (int i = 0; i < n; i++) {
        const ckksmi_direction d = t[i];
        if (check_sizes(d.rows, d.cols)) return CKKSMI_EINVAL;
        out.push_back(SeriesTensor{d.out, nullptr, d.in, nullptr, d.rows, d.cols, 1.0});
    }
    return CKKSMI_OK;
}

int muon_call(const ckksmi_muon *opt, const ckksmi_muon_tensor *t, int n, ckksmi_muon &o, std::vector<SeriesTensor> &out, bool &copies) {
    if (!opt || n < 0 || (!t && n)) return CKKSMI_EINVAL;
    o = *opt;
    const int rc = check_series(o.series);
    if (rc) return rc;
    if (!dtype_ok(o.p_dtype) || !dtype_ok(o.grad_dtype) || !(o.momentum >= 0 && o.momentum < 1) || !std::isfinite(o.lr) || !std::isfinite(o.weight_decay) ||
        !std::isfinite(o.grad_scale) || !aligned(o.skip, 4))
        return CKKSMI_EINVAL;
    copies = false;
    for (int i = 0; i < n; i++) {
        const ckksmi_muon_tensor x = t[i];
        if (check_sizes(x.rows, x.cols) || !std::isfinite(x.scale)) return CKKSMI_EINVAL;
        out.push_back(SeriesTensor{x.p, x.copy, x.grad, x.m, x.rows, x.cols, o.lr * x.scale});
        copies = copies || (x.rows && x.cols && x.copy);
    }
    return !copies || o.copy_dtype == CKKSMI_BF16 || o.copy_dtype == CKKSMI_F16 ? CKKSMI_OK : CKKSMI_EINVAL;
}

// no exception leaves an entry point
template <class F> int guarded(F f) {
    try {
        return f();
    } catch (...) {
        return CKKSMI_EUNSUPPORTED;
    }
}

}  // namespace

extern "C" int ckksmi_orthogonalise_workspace_bytes(const ckksmi_ctx *c, const ckksmi_series *s, const ckksmi_direction *t, int n, int dtype, size_t *bytes) {
    if (!c || !bytes) return CKKSMI_EINVAL;
    return guarded([&]() -> int {
        ckksmi_series series;
        std::vector<SeriesTensor> tensors;
        const int rc = directions_call(s, t, n, dtype, series, tensors);
        if (!rc) *bytes = SeriesCall(tensors, series).need;
        return rc;
    });
}

extern "C" int ckksmi_orthogonalise(ckksmi_ctx *c, const ckksmi_series *s, const ckksmi_direction *t, int n, int dtype, void *ws, size_t ws_bytes, void *stream) {
    if (!dev_ok(c)) return CKKSMI_EDEVICE;
    return guarded([&]() -> int {
        ckksmi_series series;
        std::vector<SeriesTensor> tensors;
        const int rc = directions_call(s, t, n, dtype, series, tensors);
        if (rc) return rc;
        const SeriesCall call(tensors, series);
        if (call.t.empty()) return CKKSMI_OK;
        for (const SeriesTensor &x : call.t)
            if (!x.p || !x.g || !aligned(x.p, element_bytes(dtype)) || !aligned(x.g, element_bytes(dtype))) return CKKSMI_EINVAL;
        if (call.need && (!ws || !aligned(ws, 16))) return CKKSMI_EINVAL;
        for (size_t i = 0; i < call.t.size(); i++) {
            const size_t bytes = call.plan[i].numel * element_bytes(dtype);
            if (overlap(ws, call.need, call.t[i].p, bytes) || overlap(ws, call.need, call.t[i].g, bytes)) return CKKSMI_EINVAL;
        }
        if (ws_bytes < call.need) return CKKSMI_EWORKSPACE;
        PassArgs A;
        memset(&A, 0, sizeof(A));
        A.g_dtype = dtype; A.eps = series.eps;
        Guard guard(c);
        switch (dtype) {
            case CKKSMI_F32: run_series<float, false>(c, call, series, A, ws, S(stream)); break;
            case CKKSMI_BF16: run_series<__bf16, false>(c, call, series, A, ws, S(stream)); break;
            default: run_series<_Float16, false>(c, call, series, A, ws, S(stream)); break;
        }
        return guard.rc();
    });
}

extern "C" int ckksmi_muon_workspace_bytes(const ckksmi_ctx *c, const ckksmi_muon *opt, const ckksmi_muon_tensor *t, int n, size_t *bytes) {
    if (!c || !bytes) return CKKSMI_EINVAL;
    return guarded([&]() -> int {
        ckksmi_muon o;
        std::vector<SeriesTensor> tensors;
        bool copies;
        const int rc = muon_call(opt, t, n, o, tensors, copies);
        if (!rc) *bytes = SeriesCall(tensors, o.series).need;
        return rc;
    });
}

extern "C" int ckksmi_muon_step(ckksmi_ctx *c, const ckksmi_muon *opt, const ckksmi_muon_tensor *t, int n, void *ws, size_t ws_bytes, void *stream) {
    if (!dev_ok(c)) return CKKSMI_EDEVICE;
    return guarded([&]() -> int {
        ckksmi_muon o;
        std::vector<SeriesTensor> tensors;
        bool copies;
        const int rc = muon_call(opt, t, n, o, tensors, copies);
        if (rc) return rc;
        const SeriesCall call(tensors, o.series);
        if (call.t.empty()) return CKKSMI_OK;
        const size_t ps = element_bytes(o.p_dtype), gs = element_bytes(o.grad_dtype);
        for (const SeriesTensor &x : call.t)
            if (!x.p || !x.g || !x.m || !aligned(x.p, ps) || !aligned(x.g, gs) || !aligned(x.m, 4) || !aligned(x.copy, 2)) return CKKSMI_EINVAL;
        if (call.need && (!ws || !aligned(ws, 16))) return CKKSMI_EINVAL;
        for (size_t i = 0; i < call.t.size(); i++) {
            const SeriesTensor &x = call.t[i];
            const size_t e = call.plan[i].numel;
            if (overlap(ws, call.need, x.p, e * ps) || overlap(ws, call.need, x.g, e * gs) || overlap(ws, call.need, x.m, e * 4) || overlap(ws, call.need, x.copy, e * 2))
                return CKKSMI_EINVAL;
        }
        if (ws_bytes < call.need) return CKKSMI_EWORKSPACE;
        PassArgs A;
        memset(&A, 0, sizeof(A));
        A.g_dtype = o.grad_dtype; A.copy_f16 = o.copy_dtype == CKKSMI_F16; A.nesterov = o.nesterov != 0;
        A.momentum = (float)o.momentum; A.rest = (float)(1.0 - o.momentum); A.grad_scale = (float)o.grad_scale; A.decay = (float)(1.0 - o.lr * o.weight_decay);
        A.eps = o.series.eps; A.skip = o.skip;
        Guard guard(c);
        switch (o.p_dtype) {
            case CKKSMI_F32: run_series<float, true>(c, call, o.series, A, ws, S(stream)); break;
            case CKKSMI_BF16: run_series<__bf16, true>(c, call, o.series, A, ws, S(stream)); break;
            default: run_series<_Float16, true>(c, call, o.series, A, ws, S(stream)); break;
        }
        return guard.rc();
    });
}
