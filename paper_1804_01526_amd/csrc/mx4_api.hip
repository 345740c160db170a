// Host side of the microscaled 4-bit operators and of the norm: geometry, argument validation, dispatch.  Every check runs before
// anything is queued.
#include <math.h>
#include <string.h>

#include "mx4.h"
#include "serve.h"

using namespace hbfp;

namespace {

bool known_type(int dtype) { return dtype == HBFP_F32 || dtype == HBFP_BF16 || dtype == HBFP_F16; }
int64_t size_of(int dtype) { return dtype == HBFP_F32 ? 4 : 2; }
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

int check_mx4(const hbfp_mx4 *t) {
    if (!t) return HBFP_ERR_ARG;
    hbfp_mx4 p;
    if (hbfp_mx4_plan(t->rows, t->kdim, &p) != HBFP_OK) return HBFP_ERR_LAYOUT;
    if (p.groups != t->groups || p.scale_rows != t->scale_rows || p.code_bytes != t->code_bytes || p.scale_bytes != t->scale_bytes) return HBFP_ERR_LAYOUT;
    return !t->codes || !t->scales || (((uintptr_t)t->codes | (uintptr_t)t->scales) & 15) ? HBFP_ERR_ARG : HBFP_OK;
}
Mx4View view_of(const hbfp_mx4 &t) { return {t.codes, t.scales, t.rows, t.kdim, t.groups, t.scale_rows}; }

// what a call reads or writes: `rows` rows of `width` bytes, `pitch` apart
struct Span {
    const void *at;
    uint64_t rows, width, pitch;
};
Span matrix(const void *p, int dtype, int64_t rows, int64_t cols, int64_t ld) {
    return {p, (uint64_t)rows, (uint64_t)(cols * size_of(dtype)), (uint64_t)(ld * size_of(dtype))};
}
Span bytes_at(const void *p, uint64_t n) { return {p, 1, n, n}; }
// whether two of them share a byte (columns of one matrix, at equal pitches, do not); different pitches: whether their ranges meet
bool overlap(const Span &x, const Span &y) {
    if (!x.at || !y.at) return false;
    const uint64_t a = (uint64_t)(uintptr_t)x.at, b = (uint64_t)(uintptr_t)y.at;
    const uint64_t a_end = a + (x.rows - 1) * x.pitch + x.width, b_end = b + (y.rows - 1) * y.pitch + y.width;
    if (a >= b_end || b >= a_end) return false;
    if (x.rows == 1 || y.rows == 1 || x.pitch != y.pitch) {
        // a single row against the rows of the other: it meets one unless it lies within a gap
        const Span &one = x.rows == 1 ? x : y, &many = x.rows == 1 ? y : x;
        if (one.rows != 1 || many.rows == 1) return true;
        const uint64_t o = (uint64_t)(uintptr_t)one.at, m = (uint64_t)(uintptr_t)many.at;
        if (o < m) return true;                              // (it reaches the first row, or it would end before)
        const uint64_t off = (o - m) % many.pitch;
        return off < many.width || off + one.width > many.pitch;
    }
    const uint64_t off = (a < b ? b - a : a - b) % x.pitch;  // of the later one's rows, from the earlier one's
    const uint64_t first = a < b ? x.width : y.width, second = a < b ? y.width : x.width;
    return off < first || off + second > x.pitch;
}

int check_matrix(const void *p, int dtype, int64_t rows, int64_t cols, int64_t ld) {
    if (!p || rows <= 0 || cols <= 0 || rows > 0x7fffffff || cols > 0x7fffff00 || ld < cols || ld > ((int64_t)1 << 60) / rows) return HBFP_ERR_ARG;
    if (!known_type(dtype)) return HBFP_ERR_FORMAT;
    return (uintptr_t)p & (size_of(dtype) - 1) ? HBFP_ERR_ARG : HBFP_OK;
}

int check_product(int64_t M, int64_t N, int64_t K) {
    return M <= 0 || N <= 0 || K <= 0 || M > 0x7fffffff || N > 0x7fffffff || K > 0x7fffff00 ? HBFP_ERR_ARG : HBFP_OK;
}
int64_t groups_of(int64_t K) { return ceil_div(K, 256); }

// everything of a norm call that does not depend on the form of its result
int check_norm(const hbfp_norm *n, const Span *codes, int ncodes) {
    int rc;
    if ((rc = check_matrix(n->x, n->dtype, n->rows, n->cols, n->ldx)) != HBFP_OK) return rc;
    const Span x = matrix(n->x, n->dtype, n->rows, n->cols, n->ldx), residual = matrix(n->residual, n->dtype, n->rows, n->cols, n->ld_residual);
    const Span sum = matrix(n->sum, n->dtype, n->rows, n->cols, n->ld_sum), values = matrix(n->values, n->dtype, n->rows, n->cols, n->ld_values);
    if (n->residual && (rc = check_matrix(n->residual, n->dtype, n->rows, n->cols, n->ld_residual)) != HBFP_OK) return rc;
    if (n->sum && (rc = check_matrix(n->sum, n->dtype, n->rows, n->cols, n->ld_sum)) != HBFP_OK) return rc;
    if (n->values && (rc = check_matrix(n->values, n->dtype, n->rows, n->cols, n->ld_values)) != HBFP_OK) return rc;
    if (((uintptr_t)n->weight | (uintptr_t)n->rstd) & 3) return HBFP_ERR_ARG;
    if (!(n->eps > 0.0f) || isinf(n->eps)) return HBFP_ERR_ARG;
    const Span weight = bytes_at(n->weight, 4 * (uint64_t)n->cols), rstd = bytes_at(n->rstd, 4 * (uint64_t)n->rows);
    const Span in[3] = {x, residual, weight};
    Span out[5] = {sum, values, rstd};
    int outs = 3;
    for (int i = 0; i < ncodes; ++i) out[outs++] = codes[i];
    for (int i = 0; i < outs; ++i) {
        for (int j = 0; j < 3; ++j) {
            const bool in_place = i == 0 && j < 2 && out[0].at == in[j].at && out[0].pitch == in[j].pitch;
            if (!in_place && overlap(out[i], in[j])) return HBFP_ERR_ARG;
        }
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return HBFP_ERR_ARG;
    }
    return HBFP_OK;
}

}  // namespace

extern "C" {

int hbfp_mx4_plan(int64_t rows, int64_t kdim, hbfp_mx4 *out) {
    if (!out || rows <= 0 || kdim <= 0 || rows > 0x7fffffff || kdim > 0x7fffff00) return HBFP_ERR_ARG;
    memset(out, 0, sizeof *out);
    out->rows = rows;
    out->kdim = kdim;
    out->groups = groups_of(kdim);
    out->scale_rows = round_up(rows, 16);
    out->code_bytes = (uint64_t)out->groups * (uint64_t)rows * 128;
    out->scale_bytes = (uint64_t)out->groups * (uint64_t)out->scale_rows * 8;
    return HBFP_OK;
}

int hbfp_quant_mx4(const void *src, int dtype, int64_t rows, int64_t cols, int64_t ld, int rounding, uint64_t seed,
                   const hbfp_mx4 *along, const hbfp_mx4 *down, void *stream) {
    int rc = check_matrix(src, dtype, rows, cols, ld);
    if (rc != HBFP_OK) return rc;
    if (rounding != HBFP_RNE && rounding != HBFP_STOCHASTIC) return HBFP_ERR_FORMAT;
    if (!along && !down) return HBFP_ERR_ARG;
    Mx4View a, d;
    Span out[4];
    int outs = 0;
    if (along) {
        if ((rc = check_mx4(along)) != HBFP_OK) return rc;
        if (along->rows != rows || along->kdim != cols) return HBFP_ERR_LAYOUT;
        a = view_of(*along);
        out[outs++] = bytes_at(along->codes, along->code_bytes);
        out[outs++] = bytes_at(along->scales, along->scale_bytes);
    }
    if (down) {
        if ((rc = check_mx4(down)) != HBFP_OK) return rc;
        if (down->rows != cols || down->kdim != rows) return HBFP_ERR_LAYOUT;
        d = view_of(*down);
        out[outs++] = bytes_at(down->codes, down->code_bytes);
        out[outs++] = bytes_at(down->scales, down->scale_bytes);
    }
    const Span in = matrix(src, dtype, rows, cols, ld);
    for (int i = 0; i < outs; ++i) {
        if (overlap(out[i], in)) return HBFP_ERR_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return HBFP_ERR_ARG;
    }
    return launch_quant_mx4(src, dtype, rows, cols, ld, rounding, seed, along ? &a : nullptr, down ? &d : nullptr, (hipStream_t)stream);
}

int hbfp_read_mx4(const hbfp_mx4 *t, int dtype, void *dst, int64_t ld, void *stream) {
    int rc = check_mx4(t);
    if (rc != HBFP_OK) return rc;
    if (dtype != HBFP_F32 && dtype != HBFP_BF16) return HBFP_ERR_FORMAT;
    if ((rc = check_matrix(dst, dtype, t->rows, t->kdim, ld)) != HBFP_OK) return rc;
    const Span out = matrix(dst, dtype, t->rows, t->kdim, ld);
    if (overlap(out, bytes_at(t->codes, t->code_bytes)) || overlap(out, bytes_at(t->scales, t->scale_bytes))) return HBFP_ERR_ARG;
    return launch_read_mx4(view_of(*t), dtype, dst, ld, (hipStream_t)stream);
}

int hbfp_gemm_mx4_workspace(int64_t M, int64_t N, int64_t K, size_t *bytes) {
    const int rc = check_product(M, N, K);
    if (rc != HBFP_OK || !bytes) return HBFP_ERR_ARG;
    *bytes = align256(gemm_mx4_workspace(M, N, groups_of(K)));
    return HBFP_OK;
}

int hbfp_gemm_mx4(const hbfp_mx4 *a, const hbfp_mx4 *b, const float *bias, void *y, int dtype, int64_t ldy, void *workspace,
                  size_t ws_bytes, void *stream) {
    int rc;
    if ((rc = check_mx4(a)) != HBFP_OK || (rc = check_mx4(b)) != HBFP_OK) return rc;
    if (a->kdim != b->kdim) return HBFP_ERR_LAYOUT;
    if ((rc = check_matrix(y, dtype, a->rows, b->rows, ldy)) != HBFP_OK) return rc;
    if ((uintptr_t)bias & 3) return HBFP_ERR_ARG;
    const Span out = matrix(y, dtype, a->rows, b->rows, ldy);
    const Span in[5] = {bytes_at(a->codes, a->code_bytes), bytes_at(a->scales, a->scale_bytes), bytes_at(b->codes, b->code_bytes),
                        bytes_at(b->scales, b->scale_bytes), bytes_at(bias, 4 * (uint64_t)b->rows)};
    for (const Span &i : in)
        if (overlap(out, i)) return HBFP_ERR_ARG;
    if (!gemm_mx4_fits(a->rows, b->rows, a->groups)) return HBFP_ERR_ARG;
    const size_t need = align256(gemm_mx4_workspace(a->rows, b->rows, a->groups));
    if (need && (!workspace || ws_bytes < need || ((uintptr_t)workspace & 255))) return HBFP_ERR_WORKSPACE;
    const Mx4Product p = {view_of(*a), view_of(*b), bias, y, ldy, dtype};
    return launch_gemm_mx4(p, workspace, (hipStream_t)stream);
}

int hbfp_linear_mx4_workspace(int64_t M, int64_t N, int64_t K, size_t *bytes) {
    const int rc = check_product(M, N, K);
    if (rc != HBFP_OK || !bytes) return HBFP_ERR_ARG;
    hbfp_mx4 x;
    hbfp_mx4_plan(M, K, &x);
    *bytes = linear_mx4_fused_ok(M, N, x.groups) ? 0 : align256(x.code_bytes) + align256(x.scale_bytes) + align256(gemm_mx4_workspace(M, N, x.groups));
    return HBFP_OK;
}

int hbfp_linear_mx4(const void *x, int dtype, int64_t M, int64_t ldx, const hbfp_mx4 *w, const float *bias, void *y, int64_t ldy,
                    void *workspace, size_t ws_bytes, void *stream) {
    int rc = check_mx4(w);
    if (rc != HBFP_OK) return rc;
    const int64_t K = w->kdim, N = w->rows;
    if ((rc = check_matrix(x, dtype, M, K, ldx)) != HBFP_OK) return rc;
    if ((rc = check_matrix(y, dtype, M, N, ldy)) != HBFP_OK) return rc;
    if ((uintptr_t)bias & 3) return HBFP_ERR_ARG;
    const Span out = matrix(y, dtype, M, N, ldy);
    const Span in[3] = {bytes_at(w->codes, w->code_bytes), bytes_at(w->scales, w->scale_bytes), bytes_at(bias, 4 * (uint64_t)N)};
    for (const Span &i : in)
        if (overlap(out, i)) return HBFP_ERR_ARG;
    hbfp_mx4 codes;
    hbfp_mx4_plan(M, K, &codes);
    Mx4Product p = {view_of(codes), view_of(*w), bias, y, ldy, dtype};
    if (linear_mx4_fused_ok(M, N, codes.groups)) {
        // every workgroup reads all of x for itself, while others store their part of y
        if (overlap(out, matrix(x, dtype, M, K, ldx))) return HBFP_ERR_ARG;
        return launch_linear_mx4_fused(p, x, ldx, (hipStream_t)stream);
    }
    if (!gemm_mx4_fits(M, N, codes.groups)) return HBFP_ERR_ARG;
    size_t need = 0;
    if ((rc = hbfp_linear_mx4_workspace(M, N, K, &need)) != HBFP_OK) return rc;
    if (!workspace || ws_bytes < need || ((uintptr_t)workspace & 255)) return HBFP_ERR_WORKSPACE;
    p.a.codes = (uint8_t *)workspace;
    p.a.scales = p.a.codes + align256(codes.code_bytes);
    void *const rest = p.a.scales + align256(codes.scale_bytes);
    if ((rc = launch_quant_mx4(x, dtype, M, K, ldx, HBFP_RNE, 0, &p.a, nullptr, (hipStream_t)stream)) != HBFP_OK) return rc;
    return launch_gemm_mx4(p, rest, (hipStream_t)stream);
}

int hbfp_norm_i8(const hbfp_norm *norm, int8_t *codes, float *scales, void *stream) {
    if (!norm || !codes || !scales || ((uintptr_t)codes & 15) || ((uintptr_t)scales & 3)) return HBFP_ERR_ARG;
    if (norm->rows <= 0 || norm->cols <= 0) return HBFP_ERR_ARG;
    const int64_t kpad = round_up(norm->cols, 128);
    const Span out[2] = {bytes_at(codes, (uint64_t)norm->rows * (uint64_t)kpad), bytes_at(scales, 4 * (uint64_t)norm->rows)};
    const int rc = check_norm(norm, out, 2);
    if (rc != HBFP_OK) return rc;
    const NormArgs a = {*norm, codes, scales, kpad, {}};
    return launch_norm(a, (hipStream_t)stream);
}

int hbfp_norm_mx4(const hbfp_norm *norm, const hbfp_mx4 *out, void *stream) {
    if (!norm) return HBFP_ERR_ARG;
    int rc = check_mx4(out);
    if (rc != HBFP_OK) return rc;
    if (out->rows != norm->rows || out->kdim != norm->cols) return HBFP_ERR_LAYOUT;
    const Span to[2] = {bytes_at(out->codes, out->code_bytes), bytes_at(out->scales, out->scale_bytes)};
    if ((rc = check_norm(norm, to, 2)) != HBFP_OK) return rc;
    const NormArgs a = {*norm, nullptr, nullptr, 0, view_of(*out)};
    return launch_norm(a, (hipStream_t)stream);
}

int hbfp_norm_grad_workspace(int64_t rows, int64_t cols, size_t *bytes) {
    if (!bytes || rows <= 0 || cols <= 0 || rows > 0x7fffffff || cols > 0x7fffff00) return HBFP_ERR_ARG;
    *bytes = align256(norm_grad_workspace(rows, cols));
    return HBFP_OK;
}

int hbfp_norm_grad(const void *g, int64_t ldg, const void *sum, int64_t ld_sum, const float *rstd, const float *weight, const void *g_sum,
                   int64_t ld_g_sum, int dtype, int64_t rows, int64_t cols, void *dx, int64_t ldx, float *dweight, void *workspace,
                   size_t ws_bytes, void *stream) {
    int rc;
    if ((rc = check_matrix(g, dtype, rows, cols, ldg)) != HBFP_OK || (rc = check_matrix(sum, dtype, rows, cols, ld_sum)) != HBFP_OK) return rc;
    if ((rc = check_matrix(dx, dtype, rows, cols, ldx)) != HBFP_OK) return rc;
    if (g_sum && (rc = check_matrix(g_sum, dtype, rows, cols, ld_g_sum)) != HBFP_OK) return rc;
    if (!rstd || (((uintptr_t)rstd | (uintptr_t)weight | (uintptr_t)dweight) & 3)) return HBFP_ERR_ARG;
    const Span in[5] = {matrix(g, dtype, rows, cols, ldg), matrix(g_sum, dtype, rows, cols, ld_g_sum), matrix(sum, dtype, rows, cols, ld_sum),
                        bytes_at(rstd, 4 * (uint64_t)rows), bytes_at(weight, 4 * (uint64_t)cols)};
    const Span out[2] = {matrix(dx, dtype, rows, cols, ldx), bytes_at(dweight, 4 * (uint64_t)cols)};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 5; ++j) {
            const bool in_place = i == 0 && j < 2 && out[0].at == in[j].at && out[0].pitch == in[j].pitch;
            if (!in_place && overlap(out[i], in[j])) return HBFP_ERR_ARG;
        }
    if (overlap(out[0], out[1])) return HBFP_ERR_ARG;
    const size_t need = dweight ? align256(norm_grad_workspace(rows, cols)) : 0;
    if (need && (!workspace || ws_bytes < need || ((uintptr_t)workspace & 255))) return HBFP_ERR_WORKSPACE;
    const NormGradArgs a = {g, sum, g_sum, rstd, weight, dx, dweight, (float *)workspace, ldg, ld_sum, ld_g_sum, ldx, rows, cols, dtype};
    return launch_norm_grad(a, (hipStream_t)stream);
}

}  // extern "C"
