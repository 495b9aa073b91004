// Answers from matrices in 4 bits (include/ckksmi_train.h): argument checks and launches.
#include "train_call.h"
#include "train_rows4.h"

namespace {

constexpr int64_t kMaxRows4 = 1 << 21;  // (64 rows a workgroup along y, of which a launch has 65535)

int check_matrix4(const ckksmi_matrix4 &m) {
    if (!dtype_ok(m.dtype) || m.group < 32 || m.group > 1024 || (m.group & (m.group - 1))) return CKKSMI_EINVAL;
    return m.d_in < 1 || m.d_in > kMaxDim || m.d_out < 1 || m.d_out > kMaxDim ? CKKSMI_EINVAL : CKKSMI_OK;
}
struct Weights4 { const void *codes, *scales; };
struct Sizes4 {  // a matrix's rows and bytes
    size_t ldc, lds, codes, scales, elements;
    explicit Sizes4(const ckksmi_matrix4 &m)
        : ldc(round_up((size_t)m.d_in, 32) / 2), lds(((size_t)m.d_in + m.group - 1) / m.group), codes(ldc * m.d_out), scales(lds * m.d_out * element_bytes(m.dtype)),
          elements((size_t)m.d_in * m.d_out) {}
};
inline int shift_of(int group) {
    int s = 0;
    while (32 << s < group) s++;
    return s;
}

template <class T, class O, bool XF32, int PARTS, bool GATE, int EACH> void launch_rows4(ckksmi_ctx *c, const Rows4Args &R, hipStream_t st) {
    const int blocks = (R.N + 15) / 16, tiles = (R.M + 15) / 16;
    const double flops = 2.0 * R.M * R.N * R.K * (GATE ? 2 : 1);
    const int mt = tiles <= 1 ? 1 : tiles <= 2 ? 2 : 4;
    const dim3 grid(blocks, (tiles + mt - 1) / mt);
    switch (mt) {
        case 1:
            // (one row, 8192 -> 16384: 22.7 us with four waves, 24.0 with eight, 28.8 with sixteen; 4096 -> 4096 7.0, 6.6, 7.0; 16 f32 rows 12.8, 10.6, 10.7)
            if (blocks <= 512) KL(c, CKKSMI_K_ROWS4, flops, (rows4_kernel<T, O, XF32, PARTS, GATE, 1, 8, EACH>), grid, dim3(512), st, R);
            else KL(c, CKKSMI_K_ROWS4, flops, (rows4_kernel<T, O, XF32, PARTS, GATE, 1, 4, EACH>), grid, dim3(256), st, R);
            break;
        case 2: KL(c, CKKSMI_K_ROWS4, flops, (rows4_kernel<T, O, XF32, PARTS, GATE, 2, 8, EACH>), grid, dim3(512), st, R); break;
        default: KL(c, CKKSMI_K_ROWS4, flops, (rows4_kernel<T, O, XF32, PARTS, GATE, 4, 8, EACH>), grid, dim3(512), st, R); break;
    }
}
template <class T, class O, bool XF32, int PARTS, bool GATE> void launch_rows4(ckksmi_ctx *c, const Rows4Args &R, hipStream_t st) {
    switch (R.group_shift) {
        case 0: launch_rows4<T, O, XF32, PARTS, GATE, 1>(c, R, st); break;
        case 1: launch_rows4<T, O, XF32, PARTS, GATE, 2>(c, R, st); break;
        default: launch_rows4<T, O, XF32, PARTS, GATE, 4>(c, R, st); break;
    }
}

// the product of a call's own x, or the block's first two
template <bool GATE> void rows4_of_x(ckksmi_ctx *c, int dtype, const Rows4Args &R, hipStream_t st) {
    switch (dtype) {
        case CKKSMI_F32: launch_rows4<__bf16, float, true, 3, GATE>(c, R, st); break;
        case CKKSMI_BF16: launch_rows4<__bf16, __bf16, false, 1, GATE>(c, R, st); break;
        default: launch_rows4<_Float16, _Float16, false, 1, GATE>(c, R, st); break;
    }
}
// the block's last product: h in bf16 parts
void rows4_of_h(ckksmi_ctx *c, int dtype, const Rows4Args &R, hipStream_t st) {
    switch (dtype) {
        case CKKSMI_F32: launch_rows4<__bf16, float, false, 3, false>(c, R, st); break;
        case CKKSMI_BF16: launch_rows4<__bf16, __bf16, false, 2, false>(c, R, st); break;
        default: launch_rows4<__bf16, _Float16, false, 2, false>(c, R, st); break;
    }
}

Rows4Args rows4_args(const ckksmi_matrix4 &m, int64_t rows, const void *x, size_t ldx, const Weights4 &w) {
    const Sizes4 s(m);
    Rows4Args R;
    memset(&R, 0, sizeof(R));
    R.x = (const char *)x; R.ldx = ldx;
    R.codes[0] = (const uint8_t *)w.codes; R.scales[0] = (const char *)w.scales;
    R.ldc = s.ldc; R.lds = s.lds; R.M = (int)rows; R.N = (int)m.d_out; R.K = (int)m.d_in; R.group_shift = shift_of(m.group);
    return R;
}
void rows4_to(Rows4Args &R, void *y, size_t ld, int dtype) {
    const size_t es = element_bytes(dtype);
    R.epi.o0 = y; R.epi.ldo = ld; R.epi.N = R.N; R.epi.f32_out = dtype == CKKSMI_F32;
    R.epi.whole = R.N % 8 == 0 && aligned(y, 16) && ld * es % 16 == 0;
}

template <class W, class O> void launch_pack4(ckksmi_ctx *c, const Pack4Args &A, bool back, hipStream_t st) {
    const dim3 grid((unsigned)((A.groups + 3) / 4));
    if (back) KL(c, CKKSMI_K_PACK4, (double)A.groups * A.group, (unpack4_kernel<W, O>), grid, dim3(256), st, A);
    else KL(c, CKKSMI_K_PACK4, (double)A.groups * A.group, (pack4_kernel<W, O>), grid, dim3(256), st, A);
}
template <class W> void launch_pack4(ckksmi_ctx *c, const Pack4Args &A, int dtype, bool back, hipStream_t st) {
    switch (dtype) {
        case CKKSMI_F32: launch_pack4<W, float>(c, A, back, st); break;
        case CKKSMI_BF16: launch_pack4<W, __bf16>(c, A, back, st); break;
        default: launch_pack4<W, _Float16>(c, A, back, st); break;
    }
}
int pack4(ckksmi_ctx *c, const ckksmi_matrix4 *matrix, int w_dtype, const void *w, void *codes, void *scales, bool back, hipStream_t st) {
    if (!dev_ok(c)) return CKKSMI_EDEVICE;
    if (!matrix) return CKKSMI_EINVAL;
    const ckksmi_matrix4 m = *matrix;
    const int rc = check_matrix4(m);
    if (rc) return rc;
    const Sizes4 s(m);
    const size_t bytes = s.elements * (dtype_ok(w_dtype) ? element_bytes(w_dtype) : 0);
    if (!dtype_ok(w_dtype) || !w || !codes || !scales || !aligned(codes, 16) || !aligned(scales, element_bytes(m.dtype)) || !aligned(w, element_bytes(w_dtype))) return CKKSMI_EINVAL;
    if (overlap(w, bytes, codes, s.codes) || overlap(w, bytes, scales, s.scales) || overlap(codes, s.codes, scales, s.scales)) return CKKSMI_EINVAL;
    Pack4Args A;
    memset(&A, 0, sizeof(A));
    A.w = (const char *)w; A.w_out = (char *)w; A.codes = (uint8_t *)codes; A.scales = (char *)scales;
    A.ldc = s.ldc; A.lds = s.lds; A.K = (int)m.d_in; A.group = m.group; A.groups = (int64_t)s.lds * m.d_out;
    if ((A.groups + 3) / 4 > kMaxBlocks) return CKKSMI_EUNSUPPORTED;
    Guard guard(c);
    switch (w_dtype) {
        case CKKSMI_F32: launch_pack4<float>(c, A, m.dtype, back, st); break;
        case CKKSMI_BF16: launch_pack4<__bf16>(c, A, m.dtype, back, st); break;
        default: launch_pack4<_Float16>(c, A, m.dtype, back, st); break;
    }
    return guard.rc();
}

int check_weights4(const Weights4 &w, size_t es) { return w.codes && w.scales && aligned(w.codes, 16) && aligned(w.scales, es) ? CKKSMI_OK : CKKSMI_EINVAL; }

int check_ff4(const ckksmi_gated_ff4 &f) {
    if (f.act < CKKSMI_ACT_POLY || f.act > CKKSMI_ACT_GELU || f.rows < 0 || f.rows > kMaxRows4) return CKKSMI_EINVAL;
    for (const ckksmi_matrix4 m : {ckksmi_matrix4{f.dtype, f.group, f.d_in, f.d_hidden}, ckksmi_matrix4{f.dtype, f.group, f.d_hidden, f.d_out}})
        if (check_matrix4(m)) return CKKSMI_EINVAL;
    if ((f.ld_x != 0 && (f.ld_x < f.d_in || f.ld_x > kMaxDim)) || (f.ld_y != 0 && (f.ld_y < f.d_out || f.ld_y > kMaxDim))) return CKKSMI_EINVAL;
    return CKKSMI_OK;
}
inline int h_parts(int dtype) { return dtype == CKKSMI_F32 ? 3 : 2; }
inline size_t ff4_workspace(const ckksmi_gated_ff4 &f) { return round_up((size_t)f.rows * round_up((size_t)f.d_hidden, 8) * 2 * h_parts(f.dtype), 256); }

}  // namespace

extern "C" int ckksmi_pack4(ckksmi_ctx *c, const ckksmi_matrix4 *m, int w_dtype, const void *w, void *codes, void *scales, void *stream) {
    return pack4(c, m, w_dtype, w, codes, scales, false, S(stream));
}
extern "C" int ckksmi_unpack4(ckksmi_ctx *c, const ckksmi_matrix4 *m, int w_dtype, const void *codes, const void *scales, void *w, void *stream) {
    return pack4(c, m, w_dtype, w, (void *)codes, (void *)scales, true, S(stream));
}

extern "C" int ckksmi_product4(ckksmi_ctx *c, const ckksmi_matrix4 *matrix, int64_t rows, const void *x, int64_t ld_x, const void *codes, const void *scales, void *y, int64_t ld_y,
                               void *stream) {
    if (!dev_ok(c)) return CKKSMI_EDEVICE;
    if (!matrix) return CKKSMI_EINVAL;
    const ckksmi_matrix4 m = *matrix;
    const int rc = check_matrix4(m);
    if (rc) return rc;
    if (rows < 0 || rows > kMaxRows4 || (ld_x != 0 && (ld_x < m.d_in || ld_x > kMaxDim)) || (ld_y != 0 && (ld_y < m.d_out || ld_y > kMaxDim))) return CKKSMI_EINVAL;
    const size_t es = element_bytes(m.dtype);
    const Weights4 w{codes, scales};
    if (check_weights4(w, es)) return CKKSMI_EINVAL;
    if (rows == 0) return CKKSMI_OK;
    if (!x || !y || !aligned(x, es) || !aligned(y, es)) return CKKSMI_EINVAL;
    const Sizes4 s(m);
    const size_t lx = (size_t)(ld_x ? ld_x : m.d_in), ly = (size_t)(ld_y ? ld_y : m.d_out);
    const size_t nx = ((rows - 1) * lx + m.d_in) * es, ny = ((rows - 1) * ly + m.d_out) * es;
    if (overlap(y, ny, x, nx) || overlap(y, ny, codes, s.codes) || overlap(y, ny, scales, s.scales)) return CKKSMI_EINVAL;
    Rows4Args R = rows4_args(m, rows, x, lx * es, w);
    rows4_to(R, y, ly, m.dtype);
    Guard guard(c);
    rows4_of_x<false>(c, m.dtype, R, S(stream));
    return guard.rc();
}

extern "C" int ckksmi_gated_ff4_workspace_bytes(const ckksmi_ctx *c, const ckksmi_gated_ff4 *ff, size_t *bytes) {
    if (!c || !ff || !bytes) return CKKSMI_EINVAL;
    const ckksmi_gated_ff4 f = *ff;
    const int rc = check_ff4(f);
    if (!rc) *bytes = ff4_workspace(f);
    return rc;
}

extern "C" int ckksmi_gated_ff4_forward(ckksmi_ctx *c, const ckksmi_gated_ff4 *ff, const void *x, const void *gate_codes, const void *gate_scales, const void *up_codes,
                                        const void *up_scales, const void *down_codes, const void *down_scales, void *y, void *ws, size_t ws_bytes, void *stream) {
    if (!dev_ok(c)) return CKKSMI_EDEVICE;
    if (!ff) return CKKSMI_EINVAL;
    const ckksmi_gated_ff4 f = *ff;
    const int rc = check_ff4(f);
    if (rc) return rc;
    const Weights4 w[3] = {{gate_codes, gate_scales}, {up_codes, up_scales}, {down_codes, down_scales}};
    const size_t es = element_bytes(f.dtype);
    for (const Weights4 &v : w)
        if (check_weights4(v, es)) return CKKSMI_EINVAL;
    if (f.rows == 0) return CKKSMI_OK;
    if (!x || !y || !ws || !aligned(x, es) || !aligned(y, es) || !aligned(ws, 16)) return CKKSMI_EINVAL;
    const ckksmi_matrix4 in{f.dtype, f.group, f.d_in, f.d_hidden}, out{f.dtype, f.group, f.d_hidden, f.d_out};
    const Sizes4 si(in), so(out);
    const size_t lx = (size_t)(f.ld_x ? f.ld_x : f.d_in), ly = (size_t)(f.ld_y ? f.ld_y : f.d_out), need = ff4_workspace(f);
    const size_t nx = ((f.rows - 1) * lx + f.d_in) * es, ny = ((f.rows - 1) * ly + f.d_out) * es;
    const void *p[7] = {x, w[0].codes, w[0].scales, w[1].codes, w[1].scales, w[2].codes, w[2].scales};
    const size_t n[7] = {nx, si.codes, si.scales, si.codes, si.scales, so.codes, so.scales};
    for (int i = 0; i < 7; i++)
        if (overlap(y, ny, p[i], n[i]) || overlap(ws, need, p[i], n[i])) return CKKSMI_EINVAL;
    if (overlap(y, ny, ws, need)) return CKKSMI_EINVAL;
    if (ws_bytes < need) return CKKSMI_EWORKSPACE;
    Rows4Args R = rows4_args(in, f.rows, x, lx * es, w[0]);
    R.codes[1] = (const uint8_t *)w[1].codes; R.scales[1] = (const char *)w[1].scales;
    R.epi.act.kind = f.act;
    memcpy(R.epi.act.c, f.c, sizeof(f.c));
    R.h = (char *)ws; R.ldh = round_up((size_t)f.d_hidden, 8); R.h_apart = (size_t)f.rows * R.ldh; R.h_parts = h_parts(f.dtype);
    Rows4Args D = rows4_args(out, f.rows, ws, R.ldh * 2, w[2]);
    D.x_apart = R.h_apart * 2;
    rows4_to(D, y, ly, f.dtype);
    Guard guard(c);
    rows4_of_x<true>(c, f.dtype, R, S(stream));
    rows4_of_h(c, f.dtype, D, S(stream));
    return guard.rc();
}
