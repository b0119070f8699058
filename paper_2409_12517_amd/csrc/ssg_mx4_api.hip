// C ABI of microscaled 4-bit floating point, of the linear layer on it, and of the root-mean-square norm: argument checks, buffer layouts and the
// order of the launches.  Host code only.
#include <algorithm>
#include <cmath>

#include "ssg_check_rows.h"

namespace {

constexpr int64_t kMaxMx4K = (int64_t)1 << 24;
constexpr int64_t kMaxMx4Rows = (int64_t)1 << 26;

// rows of K quantized; transposed: from K rows of `rows`
ssg_status check_mx4_shape(const char *who, int64_t rows, int64_t K) {
    if (rows < 0 || rows > kMaxMx4Rows) return fail(SSG_ERR_SHAPE, "%s: %lld rows (0 to %lld)", who, (long long)rows, (long long)kMaxMx4Rows);
    if (K < 1 || K > kMaxMx4K) return fail(SSG_ERR_SHAPE, "%s: K = %lld (1 to %lld)", who, (long long)K, (long long)kMaxMx4K);
    return SSG_OK;
}
ssg_status check_mx4_extent(const char *who, const char *name, int64_t v) {
    return extent_ok(v) ? SSG_OK : fail(SSG_ERR_SHAPE, "%s: %s = %lld must be a positive multiple of 16", who, name, (long long)v);
}
size_t mx4_bytes(int64_t rows, int64_t K) {
    return std::max<size_t>(align256((size_t)(ssg::mx4_code_bytes(rows, K) + ssg::mx4_scale_bytes(rows, K))), 256);
}
uint8_t *mx4_codes(void *q) { return static_cast<uint8_t *>(q); }
uint8_t *mx4_scales(void *q, int64_t rows, int64_t K) { return static_cast<uint8_t *>(q) + ssg::mx4_code_bytes(rows, K); }
const uint8_t *mx4_codes(const void *q) { return static_cast<const uint8_t *>(q); }
const uint8_t *mx4_scales(const void *q, int64_t rows, int64_t K) { return static_cast<const uint8_t *>(q) + ssg::mx4_code_bytes(rows, K); }
ssg_status check_mx4_buffer(const char *who, const char *name, const void *q, size_t bytes, int64_t rows, int64_t K) {
    SSG_CHECK(check_ptr(who, name, q, 256, true));
    const size_t need = mx4_bytes(rows, K);
    if (bytes < need) return fail(SSG_ERR_WORKSPACE, "%s: %s holds %zu bytes, %zu needed", who, name, bytes, need);
    return SSG_OK;
}
ssg_status check_rule(const char *who, int rule) {
    return rule == SSG_MX_FLOOR || rule == SSG_MX_CEIL ? SSG_OK : fail(SSG_ERR_ARG, "%s: rule %d", who, rule);
}
// columns of a product, and workgroups of any form that it may run in
ssg_status check_mx4_product(const char *who, int64_t rows, int64_t N) {
    SSG_CHECK(check_mx4_extent(who, "N", N));
    if (N > kMaxMx4Rows) return fail(SSG_ERR_SHAPE, "%s: N = %lld (at most %lld)", who, (long long)N, (long long)kMaxMx4Rows);
    if ((rows / 16 + 2) * (N / 16) >= ((int64_t)1 << 31)) return fail(SSG_ERR_SHAPE, "%s: %lld rows by %lld columns are too many", who, (long long)rows, (long long)N);
    return SSG_OK;
}

ssg::Mx4RowsArgs rows_args(const void *src, ssg_dtype dt, int64_t rows, int64_t K, int64_t ld, int transposed, int rule, void *q) {
    ssg::Mx4RowsArgs a;
    a.src = src; a.codes = mx4_codes(q); a.scales = mx4_scales(q, rows, K); a.rows = rows; a.K = K; a.ld = ld;
    a.bf16 = dt == SSG_BF16; a.transposed = transposed; a.ceil = rule == SSG_MX_CEIL;
    return a;
}
ssg::Mx4GemmArgs gemm_args(const void *A, int64_t M, const void *B, int64_t N, int64_t K, void *C, ssg_dtype dt, int64_t ldc) {
    ssg::Mx4GemmArgs g;
    g.A = mx4_codes(A); g.sa = mx4_scales(A, M, K); g.B = mx4_codes(B); g.sb = mx4_scales(B, N, K);
    g.C = C; g.M = M; g.N = N; g.K = K; g.ldc = ldc; g.c_f32 = dt == SSG_F32;
    return g;
}

// of ssg_mx4_linear_bwd: dY by rows, its transpose and that of x
struct BwdLayout { size_t dy, dy_t, x_t, total; };
BwdLayout bwd_layout(int64_t M, int64_t N, int64_t K) {
    BwdLayout L;
    L.dy = 0;
    L.dy_t = L.dy + mx4_bytes(M, N);
    L.x_t = L.dy_t + mx4_bytes(N, M);
    L.total = L.x_t + mx4_bytes(K, M);
    return L;
}
ssg_status check_bwd_shape(const char *who, int64_t M, int64_t N, int64_t K) {
    if (M < 0 || M > kMaxMx4K) return fail(SSG_ERR_SHAPE, "%s: M = %lld rows (0 to %lld)", who, (long long)M, (long long)kMaxMx4K);
    SSG_CHECK(check_mx4_extent(who, "N", N));
    SSG_CHECK(check_mx4_extent(who, "K", K));
    SSG_CHECK(check_mx4_shape(who, N, K));
    SSG_CHECK(check_mx4_shape(who, K, N));
    SSG_CHECK(check_mx4_product(who, M, K));
    return check_mx4_product(who, N, K);
}

constexpr int64_t kMaxNormRows = (int64_t)1 << 31;

ssg_status check_norm(const ssg_rmsnorm_desc *d, const char *who) {
    if (!d) return fail(SSG_ERR_ARG, "%s: desc is NULL", who);
    const bool quantized = d->y_format == SSG_NORM_I8 || d->y_format == SSG_NORM_MX4;
    if (d->y_format < SSG_NORM_BF16 || d->y_format > SSG_NORM_MX4) return fail(SSG_ERR_ARG, "%s: y_format %d", who, d->y_format);
    const int64_t most = quantized ? kMaxMx4Rows : kMaxNormRows;
    if (d->T < 0 || d->T > most) return fail(SSG_ERR_SHAPE, "%s: T = %lld rows (0 to %lld)", who, (long long)d->T, (long long)most);
    if (!extent_ok(d->d) || d->d > ssg::kMaxNormWidth)
        return fail(SSG_ERR_SHAPE, "%s: d = %lld must be a positive multiple of 16 up to %lld", who, (long long)d->d, (long long)ssg::kMaxNormWidth);
    if (!dtype_ok(d->x_dtype) || !dtype_ok(d->r_dtype) || !dtype_ok(d->w_dtype))
        return fail(SSG_ERR_ARG, "%s: data types %d, %d, %d of x, the residual and w", who, d->x_dtype, d->r_dtype, d->w_dtype);
    if (d->residual != 0 && d->residual != 1) return fail(SSG_ERR_ARG, "%s: residual %d (0 or 1)", who, d->residual);
    SSG_CHECK(check_rule(who, d->rule));
    if (!(d->eps >= 0x1p-100f && d->eps <= 1.0f)) return fail(SSG_ERR_ARG, "%s: eps %g (2^-100 to 1)", who, (double)d->eps);
    if (!std::isfinite(d->w_offset)) return fail(SSG_ERR_ARG, "%s: w_offset is not a finite number", who);
    for (int r : d->reserved)
        if (r) return fail(SSG_ERR_ARG, "%s: reserved fields must be zero", who);
    return SSG_OK;
}

}  // namespace

// ---- quantization -----------------------------------------------------------------------------------------
size_t ssg_mx4_bytes(int64_t rows, int64_t K) {
    if (check_mx4_shape("ssg_mx4_bytes", rows, K) != SSG_OK) return 0;
    return mx4_bytes(rows, K);
}

ssg_status ssg_mx4_quantize(const void *src, ssg_dtype src_dtype, int64_t rows, int64_t K, int64_t ld, int transposed, ssg_mx_rule rule, void *q,
                            size_t q_bytes, void *stream) {
    const char *who = "ssg_mx4_quantize";
    SSG_CHECK(check_mx4_shape(who, rows, K));
    if (transposed != 0 && transposed != 1) return fail(SSG_ERR_ARG, "%s: transposed %d (0 or 1)", who, transposed);
    SSG_CHECK(check_rule(who, rule));
    if (transposed) {
        if (rows % 16) return fail(SSG_ERR_SHAPE, "%s: rows = %lld, the source's columns, must be a multiple of 16", who, (long long)rows);
        SSG_CHECK(check_rows_of(who, "src", src, src_dtype, rows ? K : 0, rows, ld));
    } else {
        SSG_CHECK(check_mx4_extent(who, "K", K));
        SSG_CHECK(check_rows_of(who, "src", src, src_dtype, rows, K, ld));
    }
    if (rows == 0) return SSG_OK;
    SSG_CHECK(check_mx4_buffer(who, "q", q, q_bytes, rows, K));
    SSG_CHECK(check_entry(who));
    ssg::launch_mx4_quantize(rows_args(src, src_dtype, rows, K, ld, transposed, rule, q), (hipStream_t)stream);
    return check_launch(who);
}

ssg_status ssg_mx4_dequantize(const void *q, size_t q_bytes, int64_t rows, int64_t K, void *dst, ssg_dtype dst_dtype, int64_t ld, void *stream) {
    const char *who = "ssg_mx4_dequantize";
    SSG_CHECK(check_mx4_shape(who, rows, K));
    SSG_CHECK(check_rows_of(who, "dst", dst, dst_dtype, rows, K, ld));
    if (rows == 0) return SSG_OK;
    SSG_CHECK(check_mx4_buffer(who, "q", q, q_bytes, rows, K));
    SSG_CHECK(check_entry(who));
    ssg::Mx4ValuesArgs a;
    a.codes = mx4_codes(q); a.scales = mx4_scales(q, rows, K); a.dst = dst; a.rows = rows; a.K = K; a.ld = ld; a.bf16 = dst_dtype == SSG_BF16;
    ssg::launch_mx4_dequantize(a, (hipStream_t)stream);
    return check_launch(who);
}

ssg_status ssg_mx4_pack(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t K, void *q, size_t q_bytes, void *stream) {
    const char *who = "ssg_mx4_pack";
    SSG_CHECK(check_mx4_shape(who, rows, K));
    SSG_CHECK(check_mx4_extent(who, "K", K));
    if (rows == 0) return SSG_OK;
    SSG_CHECK(check_ptr(who, "codes", codes, 8, true));
    SSG_CHECK(check_ptr(who, "scales", scales, 1, true));
    SSG_CHECK(check_mx4_buffer(who, "q", q, q_bytes, rows, K));
    SSG_CHECK(check_entry(who));
    ssg::launch_mx4_pack(codes, scales, rows, K, mx4_codes(q), mx4_scales(q, rows, K), (hipStream_t)stream);
    return check_launch(who);
}

ssg_status ssg_mx4_unpack(const void *q, size_t q_bytes, int64_t rows, int64_t K, uint8_t *codes, uint8_t *scales, void *stream) {
    const char *who = "ssg_mx4_unpack";
    SSG_CHECK(check_mx4_shape(who, rows, K));
    SSG_CHECK(check_mx4_extent(who, "K", K));
    if (rows == 0) return SSG_OK;
    SSG_CHECK(check_mx4_buffer(who, "q", q, q_bytes, rows, K));
    SSG_CHECK(check_ptr(who, "codes", codes, 8, true));
    SSG_CHECK(check_ptr(who, "scales", scales, 1, true));
    SSG_CHECK(check_entry(who));
    ssg::launch_mx4_unpack(mx4_codes(q), mx4_scales(q, rows, K), rows, K, codes, scales, (hipStream_t)stream);
    return check_launch(who);
}

// ---- products -----------------------------------------------------------------------------------------------
ssg_status ssg_mx4_gemm(const void *A, size_t A_bytes, int64_t M, const void *B, size_t B_bytes, int64_t N, int64_t K, void *C, ssg_dtype c_dtype,
                        int64_t ldc, void *stream) {
    const char *who = "ssg_mx4_gemm";
    SSG_CHECK(check_mx4_shape(who, M, K));
    SSG_CHECK(check_mx4_product(who, M, N));
    SSG_CHECK(check_rows_of(who, "C", C, c_dtype, M, N, ldc));
    if (M == 0) return SSG_OK;
    SSG_CHECK(check_mx4_buffer(who, "A", A, A_bytes, M, K));
    SSG_CHECK(check_mx4_buffer(who, "B", B, B_bytes, N, K));
    SSG_CHECK(check_entry(who));
    ssg::launch_mx4_gemm(gemm_args(A, M, B, N, K, C, c_dtype, ldc), (hipStream_t)stream);
    return check_launch(who);
}

ssg_status ssg_mx4_gemm_plan(int64_t M, int64_t N, int64_t K, ssg_gemm_plan *out) {
    const char *who = "ssg_mx4_gemm_plan";
    SSG_CHECK(check_mx4_shape(who, M, K));
    SSG_CHECK(check_mx4_product(who, M, N));
    if (M == 0) return fail(SSG_ERR_SHAPE, "%s: no rows, no kernel", who);
    if (!out) return fail(SSG_ERR_ARG, "%s: out is NULL", who);
    ssg::Mx4GemmArgs g;
    g.M = M; g.N = N; g.K = K;
    const ssg::I8Plan p = ssg::mx4_gemm_plan(g);
    *out = ssg_gemm_plan{p.tile, p.tile ? 4 : 0, 0, p.tile ? 0 : p.rows, p.tile ? 0 : p.cols, 1};
    return SSG_OK;
}

size_t ssg_mx4_linear_workspace_bytes(int64_t M, int64_t K) {
    if (check_mx4_shape("ssg_mx4_linear_workspace_bytes", M, K) != SSG_OK) return 0;
    return mx4_bytes(M, K);
}

ssg_status ssg_mx4_linear(const void *x, ssg_dtype x_dtype, int64_t M, int64_t K, int64_t ldx, ssg_mx_rule rule, const void *W, size_t W_bytes, int64_t N,
                          void *y, ssg_dtype y_dtype, int64_t ldy, void *workspace, size_t workspace_bytes, void *stream) {
    const char *who = "ssg_mx4_linear";
    SSG_CHECK(check_mx4_shape(who, M, K));
    SSG_CHECK(check_mx4_extent(who, "K", K));
    SSG_CHECK(check_mx4_product(who, M, N));
    SSG_CHECK(check_rule(who, rule));
    SSG_CHECK(check_rows_of(who, "x", x, x_dtype, M, K, ldx));
    SSG_CHECK(check_rows_of(who, "y", y, y_dtype, M, N, ldy));
    if (M == 0) return SSG_OK;
    SSG_CHECK(check_mx4_buffer(who, "W", W, W_bytes, N, K));
    SSG_CHECK(check_mx4_buffer(who, "workspace", workspace, workspace_bytes, M, K));
    SSG_CHECK(check_entry(who));
    if (ssg::mx4_token_ok(M, N, K, x_dtype == SSG_BF16)) {
        ssg::Mx4TokenArgs t;
        t.x = x; t.B = mx4_codes(W); t.sb = mx4_scales(W, N, K); t.C = y; t.N = N; t.K = K; t.ld = ldx; t.ldc = ldy;
        t.rows = (int)M; t.bf16 = x_dtype == SSG_BF16; t.c_f32 = y_dtype == SSG_F32; t.ceil = rule == SSG_MX_CEIL;
        ssg::launch_mx4_token(t, (hipStream_t)stream);
        return check_launch(who);
    }
    ssg::launch_mx4_quantize(rows_args(x, x_dtype, M, K, ldx, 0, rule, workspace), (hipStream_t)stream);
    ssg::launch_mx4_gemm(gemm_args(workspace, M, W, N, K, y, y_dtype, ldy), (hipStream_t)stream);
    return check_launch(who);
}

size_t ssg_mx4_linear_bwd_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (check_bwd_shape("ssg_mx4_linear_bwd_workspace_bytes", M, N, K) != SSG_OK) return 0;
    return bwd_layout(M, N, K).total;
}

ssg_status ssg_mx4_linear_bwd(const void *dy, ssg_dtype dy_dtype, int64_t lddy, const void *x, ssg_dtype x_dtype, int64_t ldx, int64_t M, int64_t N,
                              int64_t K, ssg_mx_rule rule, const void *Wt, size_t Wt_bytes, void *dx, ssg_dtype dx_dtype, int64_t lddx, void *dW,
                              ssg_dtype dw_dtype, int64_t lddw, void *workspace, size_t workspace_bytes, void *stream) {
    const char *who = "ssg_mx4_linear_bwd";
    SSG_CHECK(check_bwd_shape(who, M, N, K));
    SSG_CHECK(check_rule(who, rule));
    if (!dx && !dW) return fail(SSG_ERR_ARG, "%s: dx and dW are both NULL", who);
    SSG_CHECK(check_rows_of(who, "dy", dy, dy_dtype, M, N, lddy));
    if (dx) {
        SSG_CHECK(check_rows_of(who, "dx", dx, dx_dtype, M, K, lddx));
        SSG_CHECK(check_mx4_buffer(who, "Wt", Wt, Wt_bytes, K, N));
    }
    if (dW) {
        SSG_CHECK(check_rows_of(who, "dW", dW, dw_dtype, N, K, lddw));
        SSG_CHECK(check_rows_of(who, "x", x, x_dtype, M, K, ldx));
    }
    const BwdLayout L = bwd_layout(M, N, K);
    SSG_CHECK(check_ptr(who, "workspace", workspace, 256, true));
    if (workspace_bytes < L.total) return fail(SSG_ERR_WORKSPACE, "%s: workspace holds %zu bytes, %zu needed", who, workspace_bytes, L.total);
    SSG_CHECK(check_entry(who));
    uint8_t *b = static_cast<uint8_t *>(workspace);
    hipStream_t st = (hipStream_t)stream;
    const ssg::Mx4RowsArgs rows = rows_args(dy, dy_dtype, M, N, lddy, 0, rule, b + L.dy);
    if (dW && M > 0)                                         // (of no rows the product is zero)
        ssg::launch_mx4_quantize_bwd(dx ? &rows : nullptr, rows_args(dy, dy_dtype, N, M, lddy, 1, rule, b + L.dy_t),
                                     rows_args(x, x_dtype, K, M, ldx, 1, rule, b + L.x_t), st);
    else if (dx)
        ssg::launch_mx4_quantize(rows, st);
    const ssg::Mx4GemmArgs gx = gemm_args(b + L.dy, M, Wt, K, N, dx, dx_dtype, lddx), gw = gemm_args(b + L.dy_t, N, b + L.x_t, K, M, dW, dw_dtype, lddw);
    if (dx && dW) ssg::launch_mx4_gemm_pair(gx, gw, st);
    else ssg::launch_mx4_gemm(dx ? gx : gw, st);
    return check_launch(who);
}

// ---- root-mean-square norm -----------------------------------------------------------------------------------
ssg_status ssg_rmsnorm_fwd(const ssg_rmsnorm_desc *desc, const void *x, const void *residual, const void *w, void *residual_out, void *y, size_t y_bytes,
                           const float *y_scale, float *y_amax, float *rstd, void *stream) {
    const char *who = "ssg_rmsnorm_fwd";
    SSG_CHECK(check_norm(desc, who));
    const int64_t T = desc->T, d = desc->d;
    SSG_CHECK(check_rows_of(who, "x", x, (ssg_dtype)desc->x_dtype, T, d, desc->ldx));
    if (desc->residual) {
        SSG_CHECK(check_rows_of(who, "residual", residual, (ssg_dtype)desc->r_dtype, T, d, desc->ldr));
        SSG_CHECK(check_rows_of(who, "residual_out", residual_out, (ssg_dtype)desc->r_dtype, T, d, desc->ldr));
    } else if (residual || residual_out) {
        return fail(SSG_ERR_ARG, "%s: a residual is given and desc.residual is 0", who);
    }
    SSG_CHECK(check_ptr(who, "w", w, 16, false));
    SSG_CHECK(check_ptr(who, "rstd", rstd, 4, false));
    const bool e4m3 = desc->y_format == SSG_NORM_E4M3;
    SSG_CHECK(check_ptr(who, "y_scale", y_scale, 4, e4m3));
    SSG_CHECK(check_ptr(who, "y_amax", y_amax, 4, false));
    if (!e4m3 && (y_scale || y_amax)) return fail(SSG_ERR_ARG, "%s: y_scale and y_amax belong to SSG_NORM_E4M3", who);
    ssg::NormArgs a;
    if (desc->y_format == SSG_NORM_I8) {
        if (T > 0) SSG_CHECK(check_i8_buffer(who, "y", y, y_bytes, T, d));
        a.y_scales = const_cast<float *>(i8_scales(y, T, d));
    } else if (desc->y_format == SSG_NORM_MX4) {
        if (T > 0) SSG_CHECK(check_mx4_buffer(who, "y", y, y_bytes, T, d));
        a.y_scales = mx4_scales(y, T, d);
    } else {
        const int64_t unit = e4m3 ? 16 : desc->y_format == SSG_NORM_BF16 ? 8 : 4;
        if (desc->ldy < d || desc->ldy % unit != 0 || desc->ldy > ((int64_t)1 << 31))
            return fail(SSG_ERR_SHAPE, "%s: %lld elements between rows of y (at least %lld, rows start on 16 bytes)", who, (long long)desc->ldy, (long long)d);
        SSG_CHECK(check_ptr(who, "y", y, 16, T > 0));
    }
    if (T == 0) return SSG_OK;
    SSG_CHECK(check_entry(who));
    a.x = x; a.r = residual; a.w = w; a.r_out = residual_out; a.y = y; a.y_scale = y_scale; a.amax = y_amax; a.rstd = rstd;
    a.T = T; a.d = d; a.ldx = desc->ldx; a.ldr = desc->ldr; a.ldy = desc->ldy; a.x_bf16 = desc->x_dtype == SSG_BF16; a.r_bf16 = desc->r_dtype == SSG_BF16;
    a.w_bf16 = desc->w_dtype == SSG_BF16; a.form = desc->y_format; a.ceil = desc->rule == SSG_MX_CEIL; a.eps = desc->eps; a.w_offset = desc->w_offset;
    ssg::launch_norm(a, (hipStream_t)stream);
    return check_launch(who);
}

size_t ssg_rmsnorm_bwd_workspace_bytes(const ssg_rmsnorm_desc *desc) {
    if (check_norm(desc, "ssg_rmsnorm_bwd_workspace_bytes") != SSG_OK) return 0;
    return align256((size_t)(ssg::norm_bwd_blocks(desc->T, desc->d) * desc->d) * 4);
}

ssg_status ssg_rmsnorm_bwd(const ssg_rmsnorm_desc *desc, const void *dy, ssg_dtype dy_dtype, int64_t lddy, const void *s, const float *rstd, const void *w,
                           const void *ds, void *dx, void *dresidual, float *dw, void *workspace, size_t workspace_bytes, void *stream) {
    const char *who = "ssg_rmsnorm_bwd";
    SSG_CHECK(check_norm(desc, who));
    const int64_t T = desc->T, d = desc->d, lds = desc->residual ? desc->ldr : desc->ldx;
    const ssg_dtype s_dtype = (ssg_dtype)(desc->residual ? desc->r_dtype : desc->x_dtype);
    SSG_CHECK(check_rows_of(who, "dy", dy, dy_dtype, T, d, lddy));
    SSG_CHECK(check_rows_of(who, "s", s, s_dtype, T, d, lds));
    SSG_CHECK(check_ptr(who, "rstd", rstd, 4, T > 0));
    SSG_CHECK(check_ptr(who, "w", w, 16, false));
    if (!desc->residual && (ds || dresidual)) return fail(SSG_ERR_ARG, "%s: ds or dresidual is given and desc.residual is 0", who);
    if (!dx && !dresidual && !dw && T > 0) return fail(SSG_ERR_ARG, "%s: dx, dresidual and dw are all NULL", who);
    if (!w && dw) return fail(SSG_ERR_ARG, "%s: dw is given and w is NULL", who);
    SSG_CHECK(check_ptr(who, "ds", ds, 16, false));
    if (dx) SSG_CHECK(check_rows_of(who, "dx", dx, (ssg_dtype)desc->x_dtype, T, d, desc->ldx));
    SSG_CHECK(check_ptr(who, "dresidual", dresidual, 16, false));
    SSG_CHECK(check_ptr(who, "dw", dw, 16, false));
    if (dw) {
        SSG_CHECK(check_ptr(who, "workspace", workspace, 16, true));
        const size_t need = ssg_rmsnorm_bwd_workspace_bytes(desc);
        if (workspace_bytes < need) return fail(SSG_ERR_WORKSPACE, "%s: workspace holds %zu bytes, %zu needed", who, workspace_bytes, need);
    }
    if (T == 0 && !dw) return SSG_OK;
    SSG_CHECK(check_entry(who));
    ssg::NormBwdArgs a;
    a.dy = dy; a.s = s; a.ds = ds; a.w = w; a.rstd = rstd; a.dx = dx; a.dr = dresidual; a.dw = dw; a.partial = static_cast<float *>(workspace);
    a.T = T; a.d = d; a.lddy = lddy; a.lds = lds; a.lddx = desc->ldx; a.dy_bf16 = dy_dtype == SSG_BF16; a.s_bf16 = s_dtype == SSG_BF16;
    a.dx_bf16 = desc->x_dtype == SSG_BF16; a.w_bf16 = desc->w_dtype == SSG_BF16; a.w_offset = desc->w_offset;
    ssg::launch_norm_bwd(a, (hipStream_t)stream);
    return check_launch(who);
}
