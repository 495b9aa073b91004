// Norms around a block (include/ckksmi_train.h): argument checks and launches.
#include "train_call.h"
#include "train_norm.h"

namespace {

constexpr int64_t kMaxNormRows = 1 << 30;  // (the kernels go on by a grid's rows from there, in 32 bits)

int check_norm(const ckksmi_residual_norm &c) {
    if (!dtype_ok(c.dtype) || (c.weight_dtype != c.dtype && c.weight_dtype != CKKSMI_F32)) return CKKSMI_EINVAL;
    for (int k : {c.pre, c.post})
        if (k < CKKSMI_NORM_NONE || k > CKKSMI_NORM_LAYER) return CKKSMI_EINVAL;
    if (c.gate < CKKSMI_GATE_NONE || c.gate > CKKSMI_GATE_ELEMENT) return CKKSMI_EINVAL;
    if (!(c.eps >= 0) || !std::isfinite(c.eps) || !std::isfinite(c.residual_scale) || !std::isfinite(c.block_scale)) return CKKSMI_EINVAL;
    if (c.rows < 0 || c.rows > kMaxNormRows || c.d < 1 || c.d > kMaxDim) return CKKSMI_EINVAL;
    for (int64_t ld : {c.ld_x, c.ld_f, c.ld_gate, c.ld_r, c.ld_n, c.ld_dr, c.ld_dn, c.ld_dx, c.ld_df, c.ld_dgate})
        if (ld != 0 && (ld < c.d || ld > kMaxDim)) return CKKSMI_EINVAL;
    return CKKSMI_OK;
}

// Threads a row (8 elements each; 16 for the longest that a forward pass holds).  Rows that no row of this table holds take the kernels for long rows
struct NormRule { int most, lanes; };
constexpr NormRule kNorm[] = {{64, 8}, {128, 16}, {256, 32}, {512, 64}, {1024, 128}, {2048, 256}, {4096, 512}, {8192, 1024}, {16384, 1024}};
constexpr int kForwardRules = 9, kBackwardRules = 8;
inline int rule_of(int64_t d, int rules) {
    int i = 0;
    while (i < rules && d > kNorm[i].most) i++;
    return i;
}
inline int threads_of(int lanes) { return lanes > 64 ? lanes : 256; }
inline int groups_of(int lanes) { return threads_of(lanes) / lanes; }

// Workgroups of a backward pass, each going through its rows: as many as the compute units hold at once, so that all have the same number of rows.
// Registers say how many: up to 168 a thread let three waves share a SIMD (768 workgroups of 256 threads).  rms norms have 145 - 168, 16-bit layer norms
// with an element's gate 164 - 168; without one, where the weights and a channel's gate are kept besides, 172 - 180: two (512)
// (16384 rows of 2048, rms, both passes: 768 172 us, 1024 209, 512 201; layer norms with a gate's columns 512 222, 768 260, an element's gate
// 768 211, 512 231)
int64_t backward_blocks(const ckksmi_residual_norm &c) {
    const int i = rule_of(c.d, kBackwardRules);
    if (i == kBackwardRules) return std::min<int64_t>(c.rows, 1024);
    const int lanes = kNorm[i].lanes, threads = threads_of(lanes), groups = groups_of(lanes);
    const bool few = (c.pre == CKKSMI_NORM_LAYER || c.post == CKKSMI_NORM_LAYER) && c.gate != CKKSMI_GATE_ELEMENT;
    const int most = lanes >= 512 ? 262144 / lanes : (few ? 512 : 768) * 256 / threads;
    return std::min<int64_t>((c.rows + groups - 1) / groups, most);
}
// waves that share the rows of a column pass, in workgroups of four
int64_t column_blocks(int64_t rows) { return std::min<int64_t>((rows + 15) / 16, 64); }
// column sums of this many go to memory
int64_t column_groups(const ckksmi_residual_norm &c) { return rule_of(c.d, kBackwardRules) == kBackwardRules ? 4 * column_blocks(c.rows) : backward_blocks(c); }
inline size_t part_ld(int64_t d) { return round_up((size_t)d, 8); }
// (never less for more rows)
size_t norm_workspace(const ckksmi_residual_norm &c) {
    const size_t part = round_up((size_t)column_groups(c) * NORM_SUMS * part_ld(c.d) * sizeof(float), 256);
    return part + (rule_of(c.d, kBackwardRules) == kBackwardRules ? (size_t)c.rows * 16 : 0);
}

struct Vectors { const void *post_w, *post_b, *pre_w, *pre_b; };

// what both passes need to know of the call: weights only where there is a norm, biases only of layer norms
int check_weights(const ckksmi_residual_norm &c, const void *f, const void *gate, const Vectors &v) {
    const size_t ws = element_bytes(c.weight_dtype), es = element_bytes(c.dtype);
    for (const void *p : {v.post_w, v.post_b, v.pre_w, v.pre_b})
        if (!aligned(p, ws)) return CKKSMI_EINVAL;
    if ((c.post == CKKSMI_NORM_NONE || !f) && (v.post_w || v.post_b)) return CKKSMI_EINVAL;
    if (c.pre == CKKSMI_NORM_NONE && (v.pre_w || v.pre_b)) return CKKSMI_EINVAL;
    if ((c.post != CKKSMI_NORM_LAYER && v.post_b) || (c.pre != CKKSMI_NORM_LAYER && v.pre_b)) return CKKSMI_EINVAL;
    if (f ? (c.gate != CKKSMI_GATE_NONE) != (gate != nullptr) : gate != nullptr) return CKKSMI_EINVAL;
    return aligned(gate, c.gate == CKKSMI_GATE_CHANNEL ? ws : es) ? CKKSMI_OK : CKKSMI_EINVAL;
}

struct Span { const void *p; size_t n; };
// bytes from the first element to the last one of a call's tensors
struct NormSpans {
    const ckksmi_residual_norm &c;
    size_t es, ws;
    explicit NormSpans(const ckksmi_residual_norm &c_) : c(c_), es(element_bytes(c_.dtype)), ws(element_bytes(c_.weight_dtype)) {}
    size_t ld(int64_t l) const { return (size_t)(l ? l : c.d) * es; }
    Span rows(const void *p, int64_t l) const { return Span{p, p ? (size_t)(c.rows - 1) * ld(l) + (size_t)c.d * es : 0}; }
    Span vector(const void *p) const { return Span{p, p ? (size_t)c.d * ws : 0}; }
    Span gate(const void *p, int64_t l) const { return c.gate == CKKSMI_GATE_ELEMENT ? rows(p, l) : vector(p); }
};
// outputs apart from inputs and from each other
bool apart(const Span *out, int n_out, const Span *in, int n_in) {
    for (int o = 0; o < n_out; o++) {
        for (int i = 0; i < n_in; i++)
            if (overlap(out[o].p, out[o].n, in[i].p, in[i].n)) return false;
        for (int i = 0; i < o; i++)
            if (overlap(out[o].p, out[o].n, out[i].p, out[i].n)) return false;
    }
    return true;
}

NormArgs norm_args(const ckksmi_residual_norm &c, const void *x, const void *f, const void *gate, const Vectors &v) {
    const NormSpans s(c);
    NormArgs A;
    memset(&A, 0, sizeof(A));
    A.x = (const char *)x; A.f = (const char *)f; A.gate = (const char *)gate;
    A.post_w = (const char *)v.post_w; A.post_b = (const char *)v.post_b; A.pre_w = (const char *)v.pre_w; A.pre_b = (const char *)v.pre_b;
    A.ld_x = s.ld(c.ld_x); A.ld_f = s.ld(c.ld_f); A.ld_gate = s.ld(c.ld_gate); A.ld_r = s.ld(c.ld_r); A.ld_n = s.ld(c.ld_n);
    A.ld_dr = s.ld(c.ld_dr); A.ld_dn = s.ld(c.ld_dn); A.ld_dx = s.ld(c.ld_dx); A.ld_df = s.ld(c.ld_df); A.ld_dgate = s.ld(c.ld_dgate);
    A.ld_part = part_ld(c.d);
    A.M = (int)c.rows; A.d = (int)c.d; A.pre = c.pre; A.post = f ? c.post : CKKSMI_NORM_NONE; A.gate_kind = f ? c.gate : CKKSMI_GATE_NONE;
    A.w_f32 = c.weight_dtype == CKKSMI_F32;
    A.eps = c.eps; A.a = f ? c.residual_scale : 1.0f; A.b = f ? c.block_scale : 0.0f; A.inv_d = (float)(1.0 / (double)c.d);
    return A;
}

template <class T, bool LAYER> void norm_forward(ckksmi_ctx *c, const NormArgs &A, int rule, dim3 grid, dim3 block, hipStream_t st) {
    const double units = (double)A.M * A.d;
    switch (rule) {
        case 0: KL(c, CKKSMI_K_NORM_FORWARD, units, (norm_forward_kernel<T, 8, 1, LAYER>), grid, block, st, A); break;
        case 1: KL(c, CKKSMI_K_NORM_FORWARD, units, (norm_forward_kernel<T, 16, 1, LAYER>), grid, block, st, A); break;
        case 2: KL(c, CKKSMI_K_NORM_FORWARD, units, (norm_forward_kernel<T, 32, 1, LAYER>), grid, block, st, A); break;
        case 3: KL(c, CKKSMI_K_NORM_FORWARD, units, (norm_forward_kernel<T, 64, 1, LAYER>), grid, block, st, A); break;
        case 4: KL(c, CKKSMI_K_NORM_FORWARD, units, (norm_forward_kernel<T, 128, 1, LAYER>), grid, block, st, A); break;
        case 5: KL(c, CKKSMI_K_NORM_FORWARD, units, (norm_forward_kernel<T, 256, 1, LAYER>), grid, block, st, A); break;
        case 6: KL(c, CKKSMI_K_NORM_FORWARD, units, (norm_forward_kernel<T, 512, 1, LAYER>), grid, block, st, A); break;
        case 7: KL(c, CKKSMI_K_NORM_FORWARD, units, (norm_forward_kernel<T, 1024, 1, LAYER>), grid, block, st, A); break;
        default: KL(c, CKKSMI_K_NORM_FORWARD, units, (norm_forward_kernel<T, 1024, 2, LAYER>), grid, block, st, A); break;
    }
}
inline bool has_layer(const NormArgs &A) { return A.pre == CKKSMI_NORM_LAYER || A.post == CKKSMI_NORM_LAYER; }
template <class T> void norm_forward(ckksmi_ctx *c, const NormArgs &A, hipStream_t st) {
    const int i = rule_of(A.d, kForwardRules);
    if (i == kForwardRules) {
        KL(c, CKKSMI_K_NORM_FORWARD, (double)A.M * A.d, (norm_forward_long_kernel<T>), dim3(std::min(A.M, 1024)), dim3(NORM_LONG), st, A);
        return;
    }
    const int threads = threads_of(kNorm[i].lanes), groups = groups_of(kNorm[i].lanes);
    // as for the backward pass: five workgroups of 256 a compute unit, of layer norms four, twice
    const int most = (has_layer(A) || threads > 256 ? 2048 : 1280) * 256 / threads;
    const dim3 grid((unsigned)std::min<int64_t>(((int64_t)A.M + groups - 1) / groups, most)), block(threads);
    if (has_layer(A)) norm_forward<T, true>(c, A, i, grid, block, st);
    else norm_forward<T, false>(c, A, i, grid, block, st);
}

template <class T> void norm_join(ckksmi_ctx *c, const NormJoinArgs &J, int outs, hipStream_t st) {
    if (outs) KL(c, CKKSMI_K_NORM_JOIN, (double)outs * J.d, (norm_join_kernel<T>), dim3((J.d + 63) / 64, outs), dim3(1024), st, J);
}

template <class T, bool LAYER, bool ELEMENT> void norm_backward(ckksmi_ctx *c, const NormArgs &A, int rule, dim3 grid, dim3 block, hipStream_t st) {
    const double units = (double)A.M * A.d;
    switch (rule) {
        case 0: KL(c, CKKSMI_K_NORM_BACKWARD, units, (norm_backward_kernel<T, 8, LAYER, ELEMENT>), grid, block, st, A); break;
        case 1: KL(c, CKKSMI_K_NORM_BACKWARD, units, (norm_backward_kernel<T, 16, LAYER, ELEMENT>), grid, block, st, A); break;
        case 2: KL(c, CKKSMI_K_NORM_BACKWARD, units, (norm_backward_kernel<T, 32, LAYER, ELEMENT>), grid, block, st, A); break;
        case 3: KL(c, CKKSMI_K_NORM_BACKWARD, units, (norm_backward_kernel<T, 64, LAYER, ELEMENT>), grid, block, st, A); break;
        case 4: KL(c, CKKSMI_K_NORM_BACKWARD, units, (norm_backward_kernel<T, 128, LAYER, ELEMENT>), grid, block, st, A); break;
        case 5: KL(c, CKKSMI_K_NORM_BACKWARD, units, (norm_backward_kernel<T, 256, LAYER, ELEMENT>), grid, block, st, A); break;
        case 6: KL(c, CKKSMI_K_NORM_BACKWARD, units, (norm_backward_kernel<T, 512, LAYER, ELEMENT>), grid, block, st, A); break;
        default: KL(c, CKKSMI_K_NORM_BACKWARD, units, (norm_backward_kernel<T, 1024, LAYER, ELEMENT>), grid, block, st, A); break;
    }
}
template <class T, bool ELEMENT> void norm_backward(ckksmi_ctx *c, NormArgs A, unsigned blocks, char *coef, hipStream_t st) {
    const int i = rule_of(A.d, kBackwardRules);
    const double units = (double)A.M * A.d;
    if (i == kBackwardRules) {
        if (A.sums) A.coef = (float *)coef;
        KL(c, CKKSMI_K_NORM_BACKWARD, units, (norm_backward_long_kernel<T, ELEMENT>), dim3(blocks), dim3(NORM_LONG), st, A);
        if (A.sums) KL(c, CKKSMI_K_NORM_BACKWARD, units, (norm_columns_kernel<T, ELEMENT>), dim3((A.d + 511) / 512, (unsigned)column_blocks(A.M)), dim3(256), st, A);
    } else {
        const dim3 grid(blocks), block(threads_of(kNorm[i].lanes));
        if (has_layer(A)) norm_backward<T, true, ELEMENT>(c, A, i, grid, block, st);
        else norm_backward<T, false, ELEMENT>(c, A, i, grid, block, st);
    }
}
template <class T> void norm_backward(ckksmi_ctx *c, const NormArgs &A, const NormJoinArgs &J, int outs, unsigned blocks, char *coef, hipStream_t st) {
    if (A.gate_kind == CKKSMI_GATE_ELEMENT) norm_backward<T, true>(c, A, blocks, coef, st);
    else norm_backward<T, false>(c, A, blocks, coef, st);
    norm_join<T>(c, J, outs, st);
}

}  // namespace

extern "C" int ckksmi_residual_norm_workspace_bytes(const ckksmi_ctx *c, const ckksmi_residual_norm *rn, size_t *bytes) {
    if (!c || !rn || !bytes) return CKKSMI_EINVAL;
    const ckksmi_residual_norm s = *rn;
    const int rc = check_norm(s);
    if (!rc) *bytes = norm_workspace(s);
    return rc;
}

extern "C" int ckksmi_residual_norm_saved_bytes(const ckksmi_ctx *c, const ckksmi_residual_norm *rn, size_t *bytes) {
    if (!c || !rn || !bytes) return CKKSMI_EINVAL;
    const ckksmi_residual_norm s = *rn;
    const int rc = check_norm(s);
    if (!rc) *bytes = (size_t)s.rows * 16;
    return rc;
}

extern "C" int ckksmi_residual_norm_forward(ckksmi_ctx *c, const ckksmi_residual_norm *rn, const void *x, const void *f, const void *gate, const void *post_w, const void *post_b,
                                            const void *pre_w, const void *pre_b, void *r, void *n, void *saved, void *stream) {
    if (!dev_ok(c)) return CKKSMI_EDEVICE;
    if (!rn) return CKKSMI_EINVAL;
    const ckksmi_residual_norm s = *rn;
    const Vectors v{post_w, post_b, pre_w, pre_b};
    int rc = check_norm(s);
    if (rc) return rc;
    if (s.rows == 0) return CKKSMI_OK;
    rc = check_weights(s, f, gate, v);
    if (rc) return rc;
    const bool pre = s.pre != CKKSMI_NORM_NONE;
    if (!x || pre != (n != nullptr) || (!pre && !r) || (!f && r)) return CKKSMI_EINVAL;
    const NormSpans at(s);
    for (const void *p : {x, f, (const void *)r, (const void *)n})
        if (!aligned(p, at.es)) return CKKSMI_EINVAL;
    if (!aligned(saved, 16)) return CKKSMI_EINVAL;
    const Span in[7] = {at.rows(x, s.ld_x), at.rows(f, s.ld_f), at.gate(gate, s.ld_gate), at.vector(post_w), at.vector(post_b), at.vector(pre_w), at.vector(pre_b)};
    const Span out[3] = {at.rows(r, s.ld_r), at.rows(n, s.ld_n), Span{saved, saved ? (size_t)s.rows * 16 : 0}};
    const bool in_place = r == x && at.ld(s.ld_r) == at.ld(s.ld_x);
    if (!apart(out, 3, in_place ? in + 1 : in, in_place ? 6 : 7)) return CKKSMI_EINVAL;
    NormArgs A = norm_args(s, x, f, gate, v);
    A.r = (char *)r; A.n = (char *)n; A.stats = (float *)saved;
    Guard guard(c);
    switch (s.dtype) {
        case CKKSMI_F32: norm_forward<float>(c, A, S(stream)); break;
        case CKKSMI_BF16: norm_forward<__bf16>(c, A, S(stream)); break;
        default: norm_forward<_Float16>(c, A, S(stream)); break;
    }
    return guard.rc();
}

extern "C" int ckksmi_residual_norm_backward(ckksmi_ctx *c, const ckksmi_residual_norm *rn, const void *x, const void *f, const void *gate, const void *post_w, const void *post_b,
                                             const void *pre_w, const void *saved, const void *dr, const void *dn, void *dx, void *df, void *dgate, void *dpost_w, void *dpost_b,
                                             void *dpre_w, void *dpre_b, int accumulate, void *ws, size_t ws_bytes, void *stream) {
    if (!dev_ok(c)) return CKKSMI_EDEVICE;
    if (!rn) return CKKSMI_EINVAL;
    const ckksmi_residual_norm s = *rn;
    const Vectors v{post_w, post_b, pre_w, nullptr};
    int rc = check_norm(s);
    if (rc) return rc;
    const NormSpans at(s);
    const bool none = s.rows == 0;  // then x, f and gate may be anything: the sums are zeros
    if (!none) {
        rc = check_weights(s, f, gate, v);
        if (rc) return rc;
        if (!x || !saved || !aligned(saved, 16)) return CKKSMI_EINVAL;
        for (const void *p : {x, f, dr, dn, (const void *)dx, (const void *)df})
            if (!aligned(p, at.es)) return CKKSMI_EINVAL;
        if (!f && (df || dgate || dpost_w || dpost_b)) return CKKSMI_EINVAL;
    }
    for (const void *p : {(const void *)dpost_w, (const void *)dpost_b, (const void *)dpre_w, (const void *)dpre_b})
        if (!aligned(p, at.ws)) return CKKSMI_EINVAL;
    if (!aligned(dgate, s.gate == CKKSMI_GATE_CHANNEL ? at.ws : at.es)) return CKKSMI_EINVAL;
    if ((s.gate == CKKSMI_GATE_NONE && dgate) || (s.post == CKKSMI_NORM_NONE && dpost_w) || (s.post != CKKSMI_NORM_LAYER && dpost_b) ||
        (s.pre == CKKSMI_NORM_NONE && (dn || dpre_w)) || (s.pre != CKKSMI_NORM_LAYER && dpre_b))
        return CKKSMI_EINVAL;
    // which column sums, and what comes of them
    const bool column_gate = s.gate == CKKSMI_GATE_CHANNEL && dgate, gated = s.gate == CKKSMI_GATE_CHANNEL, biased = s.post == CKKSMI_NORM_LAYER;
    const int sums = (dpost_w || column_gate ? SUM_P : 0) | (dpost_b || (column_gate && biased) ? SUM_Q : 0) | (dpre_w ? SUM_R : 0) | (dpre_b ? SUM_T : 0);
    NormJoinArgs J;
    memset(&J, 0, sizeof(J));
    J.d = (int)s.d; J.w_f32 = s.weight_dtype == CKKSMI_F32; J.accumulate = accumulate != 0; J.ld_part = part_ld(s.d);
    int place[NORM_SUMS], outs = 0;
    for (int k = 0; k < NORM_SUMS; k++) place[k] = sums >> k & 1 ? J.vectors++ : -1;
    auto add = [&](void *o, int first, const void *by, int second, const void *second_by) {
        if (o) J.out[outs++] = NormJoinArgs::Out{(char *)o, first, second, (const char *)by, (const char *)second_by};
    };
    add(dpost_w, place[0], gated ? gate : nullptr, -1, nullptr);
    add(dpost_b, place[1], gated ? gate : nullptr, -1, nullptr);
    add(dpre_w, place[2], nullptr, -1, nullptr);
    add(dpre_b, place[3], nullptr, -1, nullptr);
    if (column_gate) add(dgate, place[0], post_w, biased && post_b ? place[1] : -1, post_b);
    const size_t need = norm_workspace(s);
    Guard guard(c);
    if (none) {
        if (J.accumulate) return CKKSMI_OK;
        for (NormJoinArgs::Out &o : J.out) o.by = o.second_by = nullptr;
        const Span out[NORM_SUMS + 1] = {at.vector(dpost_w), at.vector(dpost_b), at.vector(dpre_w), at.vector(dpre_b), at.vector(column_gate ? dgate : nullptr)};
        if (!apart(out, NORM_SUMS + 1, nullptr, 0)) return CKKSMI_EINVAL;
    } else {
        const Span in[9] = {at.rows(x, s.ld_x), at.rows(f, s.ld_f), at.gate(gate, s.ld_gate), at.vector(post_w), at.vector(post_b), at.vector(pre_w),
                            at.rows(dr, s.ld_dr), at.rows(dn, s.ld_dn), Span{saved, (size_t)s.rows * 16}};
        const Span out[8] = {at.rows(dx, s.ld_dx), at.rows(df, s.ld_df), at.gate(dgate, s.ld_dgate), at.vector(dpost_w), at.vector(dpost_b), at.vector(dpre_w),
                             at.vector(dpre_b), Span{ws, ws && sums ? need : 0}};
        if (!apart(out, 8, in, 9)) return CKKSMI_EINVAL;
        if (sums) {
            if (!ws || !aligned(ws, 16)) return CKKSMI_EINVAL;
            if (ws_bytes < need) return CKKSMI_EWORKSPACE;
        }
    }
    NormArgs A = norm_args(s, x, f, gate, v);
    A.stats = (float *)saved; A.dr = (const char *)dr; A.dn = (const char *)dn; A.dx = (char *)dx; A.df = (char *)df;
    A.dgate = column_gate ? nullptr : (char *)dgate;
    A.sums = sums; A.vectors = J.vectors; A.part = (float *)ws;
    J.part = (const float *)ws;
    J.groups = none ? 0 : (int)column_groups(s);
    char *const coef = (char *)ws + round_up((size_t)column_groups(s) * NORM_SUMS * part_ld(s.d) * sizeof(float), 256);
    const unsigned blocks = (unsigned)backward_blocks(s);
    const hipStream_t st = S(stream);
    switch (s.dtype) {
        case CKKSMI_F32: none ? norm_join<float>(c, J, outs, st) : norm_backward<float>(c, A, J, outs, blocks, coef, st); break;
        case CKKSMI_BF16: none ? norm_join<__bf16>(c, J, outs, st) : norm_backward<__bf16>(c, A, J, outs, blocks, coef, st); break;
        default: none ? norm_join<_Float16>(c, J, outs, st) : norm_backward<_Float16>(c, A, J, outs, blocks, coef, st); break;
    }
    return guard.rc();
}
