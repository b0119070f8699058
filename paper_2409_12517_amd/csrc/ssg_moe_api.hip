// C ABI of the routing, of the products in 8-bit integers and of the layer that runs them together: argument checks, buffer
// layouts and the order of the launches.  Host code only.
#include <algorithm>
#include <cmath>

#include "ssg_check_rows.h"

namespace {

constexpr int64_t kMaxAssignments = (int64_t)1 << 26;
constexpr int kI8Align = 16;

ssg_status check_route(const ssg_route_desc *d, const char *who) {
    if (!d) return fail(SSG_ERR_ARG, "%s: desc is NULL", who);
    if (d->E < 1 || d->E > ssg::kMaxExperts) return fail(SSG_ERR_SHAPE, "%s: E = %d experts (1 to %d)", who, d->E, ssg::kMaxExperts);
    if (d->k < 1 || d->k > ssg::kMaxChosen || d->k > d->E)
        return fail(SSG_ERR_SHAPE, "%s: k = %d of %d experts (1 to %d)", who, d->k, d->E, ssg::kMaxChosen);
    if (d->T < 0 || d->T > std::min(ssg::kMaxTokens, kMaxAssignments / d->k))
        return fail(SSG_ERR_SHAPE, "%s: T = %lld tokens (0 to %lld, T k to %lld)", who, (long long)d->T, (long long)ssg::kMaxTokens, (long long)kMaxAssignments);
    if (d->ld < d->E || d->ld > ((int64_t)1 << 31)) return fail(SSG_ERR_SHAPE, "%s: ld = %lld below E = %d, or too large", who, (long long)d->ld, d->E);
    if (!dtype_ok(d->logits_dtype)) return fail(SSG_ERR_ARG, "%s: logits_dtype %d", who, d->logits_dtype);
    if (d->score != SSG_ROUTE_SOFTMAX && d->score != SSG_ROUTE_SIGMOID) return fail(SSG_ERR_ARG, "%s: score %d", who, d->score);
    if (d->groups < 1 || d->groups > ssg::kMaxGroups || d->E % d->groups != 0)
        return fail(SSG_ERR_SHAPE, "%s: groups = %d must divide E = %d and be at most %d", who, d->groups, d->E, ssg::kMaxGroups);
    if (d->top_groups < 1 || d->top_groups > d->groups || (int64_t)d->top_groups * (d->E / d->groups) < d->k)
        return fail(SSG_ERR_SHAPE, "%s: top_groups = %d of %d groups leave fewer than k = %d experts, or are none", who, d->top_groups, d->groups, d->k);
    if (d->group_top != 1 && d->group_top != 2) return fail(SSG_ERR_ARG, "%s: group_top %d (1 or 2)", who, d->group_top);
    if (d->renorm != 0 && d->renorm != 1) return fail(SSG_ERR_ARG, "%s: renorm %d (0 or 1)", who, d->renorm);
    if (!std::isfinite(d->scale)) return fail(SSG_ERR_ARG, "%s: scale is not a finite number", who);
    if (d->row_align < 1 || d->row_align > 256 || (d->row_align & (d->row_align - 1)))
        return fail(SSG_ERR_ARG, "%s: row_align %d (a power of two up to 256)", who, d->row_align);
    for (int r : d->reserved)
        if (r) return fail(SSG_ERR_ARG, "%s: reserved fields must be zero", who);
    return SSG_OK;
}

int64_t route_rows(const ssg_route_desc &d) {
    const int64_t n = d.T * d.k;
    return (n + std::min<int64_t>(d.E, n) * (d.row_align - 1)) / d.row_align * d.row_align;
}

ssg::RouteArgs route_args(const ssg_route_desc &d) {
    ssg::RouteArgs a;
    a.T = d.T; a.ld = d.ld; a.rows = route_rows(d); a.E = d.E; a.k = d.k; a.bf16 = d.logits_dtype == SSG_BF16; a.score = d.score;
    a.groups = d.groups; a.top_groups = d.top_groups; a.group_top = d.group_top; a.renorm = d.renorm; a.align = d.row_align; a.scale = d.scale;
    return a;
}

// columns of a product, and workgroups of any form that it may run in
ssg_status check_i8_product(const char *who, int64_t rows, int64_t experts, int64_t N) {
    if (!extent_ok(N) || N > kMaxI8Rows / experts) return fail(SSG_ERR_SHAPE, "%s: N = %lld must be a positive multiple of 16, at most %lld", who, (long long)N, (long long)(kMaxI8Rows / experts));
    if ((rows / 16 + 1 + experts) * (N / 16) >= ((int64_t)1 << 31)) return fail(SSG_ERR_SHAPE, "%s: %lld rows by %lld columns are too many", who, (long long)rows, (long long)N);
    return SSG_OK;
}

// whether the experts' results, the terms of the weighted sum, are fp32
bool f32_results(const ssg_moe_desc &d) { return d.y_dtype == SSG_F32 || d.f32_terms; }

struct MoeLayout { size_t ids, weights, counts, offsets, place, source, hist, tiles, x_q, h, h_q, o, total; int64_t rows; };
// words of a list of row tiles, whichever products run (no tile has fewer than 16 rows)
size_t moe_list_words(int64_t rows) { return (ssg::i8_tile_list_words(rows / 16) + 63) / 64 * 64; }
MoeLayout moe_layout(const ssg_moe_desc &d) {
    MoeLayout L;
    const ssg_route_desc &r = d.route;
    const size_t n = (size_t)r.T * r.k;
    L.rows = route_rows(r);
    size_t o = 0;
    auto take = [&](size_t bytes) { size_t at = o; o += align256(bytes); return at; };
    L.ids = take(n * 4); L.weights = take(n * 4); L.counts = take((size_t)r.E * 4); L.offsets = take(((size_t)r.E + 1) * 4);
    L.place = take(n * 4); L.source = take((size_t)L.rows * 4); L.hist = take(ssg::route_hist_bytes(route_args(r)));
    L.tiles = take(2 * moe_list_words(L.rows) * 4);
    L.x_q = take(i8_bytes(L.rows, d.d));
    L.h = take((size_t)L.rows * d.f * 2);
    L.h_q = take(i8_bytes(L.rows, d.f));
    L.o = take((size_t)L.rows * d.d * (f32_results(d) ? 4 : 2));
    L.total = o;
    return L;
}

// Up to four tokens run without an order of dispatch: a token's experts are its own.
bool few_tokens(const ssg_moe_desc &d) { return ssg::i8_mix_ok(d.route.T, d.d, d.f, d.route.k); }

ssg_status check_moe(const ssg_moe_desc *d, const char *who) {
    if (!d) return fail(SSG_ERR_ARG, "%s: desc is NULL", who);
    SSG_CHECK(check_route(&d->route, who));
    if (d->route.row_align != kI8Align) return fail(SSG_ERR_ARG, "%s: route.row_align %d (the products take %d)", who, d->route.row_align, kI8Align);
    if (!dtype_ok(d->y_dtype)) return fail(SSG_ERR_ARG, "%s: y_dtype %d", who, d->y_dtype);
    if (d->f32_terms != 0 && d->f32_terms != 1) return fail(SSG_ERR_ARG, "%s: f32_terms %d (0 or 1)", who, d->f32_terms);
    for (int r : d->reserved)
        if (r) return fail(SSG_ERR_ARG, "%s: reserved fields must be zero", who);
    const int64_t rows = route_rows(d->route);
    SSG_CHECK(check_i8_shape(who, rows, d->d));
    SSG_CHECK(check_i8_shape(who, rows, d->f));
    SSG_CHECK(check_i8_product(who, rows, d->route.E, d->f));
    return check_i8_product(who, rows, d->route.E, d->d);
}

}  // namespace

// ---- routing -------------------------------------------------------------------------------------------
size_t ssg_route_workspace_bytes(const ssg_route_desc *desc) {
    if (check_route(desc, "ssg_route_workspace_bytes") != SSG_OK) return 0;
    return std::max<size_t>(align256(ssg::route_hist_bytes(route_args(*desc))), 256);
}

int64_t ssg_route_rows(const ssg_route_desc *desc) {
    const ssg_status rc = check_route(desc, "ssg_route_rows");
    return rc == SSG_OK ? route_rows(*desc) : rc;
}

ssg_status ssg_route(const ssg_route_desc *desc, const void *logits, const float *bias, int32_t *ids, float *weights, int32_t *counts,
                     int32_t *offsets, int32_t *place, int32_t *source, void *workspace, size_t workspace_bytes, void *stream) {
    const char *who = "ssg_route";
    SSG_CHECK(check_route(desc, who));
    const bool tokens = desc->T > 0;
    SSG_CHECK(check_ptr(who, "logits", logits, desc->logits_dtype == SSG_BF16 ? 2 : 4, tokens));
    SSG_CHECK(check_ptr(who, "bias", bias, 4, false));
    SSG_CHECK(check_ptr(who, "ids", ids, 4, tokens));
    SSG_CHECK(check_ptr(who, "weights", weights, 4, tokens));
    const bool sorts = counts || offsets || place || source;
    SSG_CHECK(check_ptr(who, "counts", counts, 4, sorts));
    SSG_CHECK(check_ptr(who, "offsets", offsets, 4, sorts));
    SSG_CHECK(check_ptr(who, "place", place, 4, sorts && tokens));
    SSG_CHECK(check_ptr(who, "source", source, 4, sorts && tokens));
    ssg::RouteArgs a = route_args(*desc);
    const size_t need = sorts ? ssg::route_hist_bytes(a) : 0;
    if (need) {
        SSG_CHECK(check_ptr(who, "workspace", workspace, 16, true));
        if (workspace_bytes < need) return fail(SSG_ERR_WORKSPACE, "%s: workspace holds %zu bytes, %zu needed", who, workspace_bytes, need);
    }
    SSG_CHECK(check_entry(who));
    a.logits = logits; a.bias = bias; a.ids = ids; a.weights = weights; a.counts = counts; a.offsets = offsets; a.place = place; a.source = source;
    a.hist = static_cast<uint16_t *>(workspace);
    ssg::launch_route(a, (hipStream_t)stream);
    return check_launch(who);
}

ssg_status ssg_route_bwd(const ssg_route_desc *desc, const void *logits, const int32_t *ids, const float *weights, const float *dweights,
                         void *dlogits, void *stream) {
    const char *who = "ssg_route_bwd";
    SSG_CHECK(check_route(desc, who));
    if (desc->T == 0) return SSG_OK;
    SSG_CHECK(check_ptr(who, "logits", logits, desc->logits_dtype == SSG_BF16 ? 2 : 4, true));
    SSG_CHECK(check_ptr(who, "ids", ids, 4, true));
    SSG_CHECK(check_ptr(who, "weights", weights, 4, true));
    SSG_CHECK(check_ptr(who, "dweights", dweights, 4, true));
    SSG_CHECK(check_ptr(who, "dlogits", dlogits, 16, true));
    SSG_CHECK(check_entry(who));
    ssg::RouteBwdArgs a;
    a.logits = logits; a.ids = ids; a.weights = weights; a.dweights = dweights; a.dlogits = dlogits;
    a.T = desc->T; a.ld = desc->ld; a.E = desc->E; a.k = desc->k; a.bf16 = desc->logits_dtype == SSG_BF16; a.score = desc->score;
    a.renorm = desc->renorm; a.scale = desc->scale;
    ssg::launch_route_bwd(a, (hipStream_t)stream);
    return check_launch(who);
}

// ---- products in 8-bit integers ---------------------------------------------------------------------------
size_t ssg_i8_bytes(int64_t rows, int64_t K) {
    if (check_i8_shape("ssg_i8_bytes", rows, K) != SSG_OK) return 0;
    return i8_bytes(rows, K);
}

ssg_status ssg_i8_quantize(const void *src, ssg_dtype src_dtype, int64_t rows, int64_t K, int64_t ld, void *q, size_t q_bytes, void *stream) {
    const char *who = "ssg_i8_quantize";
    SSG_CHECK(check_i8_shape(who, rows, K));
    SSG_CHECK(check_rows_of(who, "src", src, src_dtype, rows, K, ld));
    if (rows == 0) return SSG_OK;
    SSG_CHECK(check_i8_buffer(who, "q", q, q_bytes, rows, K));
    SSG_CHECK(check_entry(who));
    ssg::I8RowsArgs a;
    a.src = src; a.codes = static_cast<uint8_t *>(q); a.scales = const_cast<float *>(i8_scales(q, rows, K));
    a.rows = rows; a.K = K; a.ld = ld; a.bf16 = src_dtype == SSG_BF16;
    ssg::launch_i8_quantize(a, (hipStream_t)stream);
    return check_launch(who);
}

ssg_status ssg_i8_pack(const int8_t *codes, const float *scales, int64_t rows, int64_t K, void *q, size_t q_bytes, void *stream) {
    const char *who = "ssg_i8_pack";
    SSG_CHECK(check_i8_shape(who, rows, K));
    if (rows == 0) return SSG_OK;
    SSG_CHECK(check_ptr(who, "codes", codes, 16, true));
    SSG_CHECK(check_ptr(who, "scales", scales, 4, true));
    SSG_CHECK(check_i8_buffer(who, "q", q, q_bytes, rows, K));
    SSG_CHECK(check_entry(who));
    ssg::launch_i8_pack(codes, scales, rows, K, static_cast<uint8_t *>(q), const_cast<float *>(i8_scales(q, rows, K)), (hipStream_t)stream);
    return check_launch(who);
}

ssg_status ssg_i8_unpack(const void *q, size_t q_bytes, int64_t rows, int64_t K, int8_t *codes, float *scales, void *stream) {
    const char *who = "ssg_i8_unpack";
    SSG_CHECK(check_i8_shape(who, rows, K));
    if (rows == 0) return SSG_OK;
    SSG_CHECK(check_i8_buffer(who, "q", q, q_bytes, rows, K));
    SSG_CHECK(check_ptr(who, "codes", codes, 16, true));
    SSG_CHECK(check_ptr(who, "scales", scales, 4, true));
    SSG_CHECK(check_entry(who));
    ssg::launch_i8_unpack(static_cast<const uint8_t *>(q), i8_scales(q, rows, K), rows, K, codes, scales, (hipStream_t)stream);
    return check_launch(who);
}

ssg_status ssg_i8_gemm(const void *A, size_t A_bytes, int64_t M, const void *B, size_t B_bytes, int64_t N, int64_t K, void *C, ssg_dtype c_dtype,
                       int64_t ldc, void *stream) {
    const char *who = "ssg_i8_gemm";
    SSG_CHECK(check_i8_shape(who, M, K));
    SSG_CHECK(check_i8_product(who, M, 1, N));
    SSG_CHECK(check_rows_of(who, "C", C, c_dtype, M, N, ldc));
    if (M == 0) return SSG_OK;
    SSG_CHECK(check_i8_buffer(who, "A", A, A_bytes, M, K));
    SSG_CHECK(check_i8_buffer(who, "B", B, B_bytes, N, K));
    SSG_CHECK(check_entry(who));
    ssg::I8GemmArgs g;
    g.A = static_cast<const uint8_t *>(A); g.sa = i8_scales(A, M, K); g.B = static_cast<const uint8_t *>(B); g.sb = i8_scales(B, N, K);
    g.C = C; g.M = M; g.N = N; g.K = K; g.ldc = ldc; g.c_f32 = c_dtype == SSG_F32;
    ssg::launch_i8_gemm(g, (hipStream_t)stream);
    return check_launch(who);
}

ssg_status ssg_i8_gemm_plan(int64_t M, int64_t N, int64_t K, int32_t experts, int swiglu, ssg_gemm_plan *out) {
    const char *who = "ssg_i8_gemm_plan";
    SSG_CHECK(check_i8_shape(who, M, K));
    if (experts < 0 || experts > ssg::kMaxExperts) return fail(SSG_ERR_SHAPE, "%s: %d experts (0 to %d)", who, experts, ssg::kMaxExperts);
    if (swiglu != 0 && swiglu != 1) return fail(SSG_ERR_ARG, "%s: swiglu %d (0 or 1)", who, swiglu);
    if (swiglu && experts == 0) return fail(SSG_ERR_UNSUPPORTED, "%s: the gate/up form is a mixture's (experts > 0)", who);
    SSG_CHECK(check_i8_product(who, M, std::max(experts, 1), N));
    if (M == 0) return fail(SSG_ERR_SHAPE, "%s: no rows, no kernel", who);
    if (!out) return fail(SSG_ERR_ARG, "%s: out is NULL", who);
    ssg::I8GemmArgs g;
    static const uint8_t some = 0;
    g.M = M; g.N = N; g.K = K; g.E = experts; g.rows_expected = M; g.B2 = swiglu ? &some : nullptr;
    const ssg::I8Plan p = ssg::i8_gemm_plan(g);
    *out = ssg_gemm_plan{p.tile, p.tile ? 4 : 0, 0, p.tile ? 0 : p.rows, p.tile ? 0 : p.cols, 1};
    return SSG_OK;
}

size_t ssg_i8_linear_workspace_bytes(int64_t M, int64_t K) {
    if (check_i8_shape("ssg_i8_linear_workspace_bytes", M, K) != SSG_OK) return 0;
    return i8_bytes(M, K);
}

ssg_status ssg_i8_linear(const void *x, ssg_dtype x_dtype, int64_t M, int64_t K, int64_t ldx, const void *W, size_t W_bytes, int64_t N, void *y,
                         ssg_dtype y_dtype, int64_t ldy, void *workspace, size_t workspace_bytes, void *stream) {
    const char *who = "ssg_i8_linear";
    SSG_CHECK(check_i8_shape(who, M, K));
    SSG_CHECK(check_i8_product(who, M, 1, N));
    SSG_CHECK(check_rows_of(who, "x", x, x_dtype, M, K, ldx));
    SSG_CHECK(check_rows_of(who, "y", y, y_dtype, M, N, ldy));
    if (M == 0) return SSG_OK;
    SSG_CHECK(check_i8_buffer(who, "W", W, W_bytes, N, K));
    SSG_CHECK(check_i8_buffer(who, "workspace", workspace, workspace_bytes, M, K));
    SSG_CHECK(check_entry(who));
    if (ssg::i8_token_ok(M, N, K)) {
        ssg::I8TokenArgs k;
        k.src = x; k.rows = (int)M; k.K = K; k.ld = ldx; k.bf16 = x_dtype == SSG_BF16;
        k.B = static_cast<const uint8_t *>(W); k.sb = i8_scales(W, N, K); k.C = y; k.N = N; k.ldc = ldy; k.c_f32 = y_dtype == SSG_F32;
        ssg::launch_i8_token(k, (hipStream_t)stream);
        return check_launch(who);
    }
    ssg::I8RowsArgs a;
    a.src = x; a.codes = static_cast<uint8_t *>(workspace); a.scales = const_cast<float *>(i8_scales(workspace, M, K));
    a.rows = M; a.K = K; a.ld = ldx; a.bf16 = x_dtype == SSG_BF16;
    ssg::I8GemmArgs g;
    g.A = a.codes; g.sa = a.scales; g.B = static_cast<const uint8_t *>(W); g.sb = i8_scales(W, N, K);
    g.C = y; g.M = M; g.N = N; g.K = K; g.ldc = ldy; g.c_f32 = y_dtype == SSG_F32;
    ssg::launch_i8_quantize(a, (hipStream_t)stream);
    ssg::launch_i8_gemm(g, (hipStream_t)stream);
    return check_launch(who);
}

// ---- the layer -------------------------------------------------------------------------------------------
size_t ssg_moe_workspace_bytes(const ssg_moe_desc *desc) {
    if (check_moe(desc, "ssg_moe_workspace_bytes") != SSG_OK) return 0;
    return moe_layout(*desc).total;
}

ssg_status ssg_moe_view_workspace(const ssg_moe_desc *desc, const void *workspace, ssg_moe_workspace_view *out) {
    SSG_CHECK(check_moe(desc, "ssg_moe_view_workspace"));
    if (!workspace || !out) return fail(SSG_ERR_ARG, "ssg_moe_view_workspace: workspace or out is NULL");
    const MoeLayout L = moe_layout(*desc);
    const uint8_t *b = static_cast<const uint8_t *>(workspace);
    out->rows = L.rows;
    out->ids = reinterpret_cast<const int32_t *>(b + L.ids);
    out->weights = reinterpret_cast<const float *>(b + L.weights);
    out->h = b + L.h;
    out->counts = out->offsets = out->place = out->source = nullptr;
    out->x_q = out->h_q = out->o = nullptr;
    if (few_tokens(*desc)) {
        out->rows = desc->route.T * desc->route.k;
        return SSG_OK;
    }
    out->counts = reinterpret_cast<const int32_t *>(b + L.counts);
    out->offsets = reinterpret_cast<const int32_t *>(b + L.offsets);
    out->place = reinterpret_cast<const int32_t *>(b + L.place);
    out->source = reinterpret_cast<const int32_t *>(b + L.source);
    out->x_q = b + L.x_q; out->h_q = b + L.h_q; out->o = b + L.o;
    return SSG_OK;
}

ssg_status ssg_moe_fwd(const ssg_moe_desc *desc, const void *x, const void *logits, const float *bias, const void *W1, size_t W1_bytes,
                       const void *W2, size_t W2_bytes, const void *W3, size_t W3_bytes, void *y, void *workspace, size_t workspace_bytes,
                       void *stream) {
    const char *who = "ssg_moe_fwd";
    SSG_CHECK(check_moe(desc, who));
    const ssg_route_desc &r = desc->route;
    if (r.T == 0) return SSG_OK;
    const int64_t d = desc->d, f = desc->f, E = r.E;
    SSG_CHECK(check_ptr(who, "x", x, 16, true));
    SSG_CHECK(check_ptr(who, "logits", logits, r.logits_dtype == SSG_BF16 ? 2 : 4, true));
    SSG_CHECK(check_ptr(who, "bias", bias, 4, false));
    SSG_CHECK(check_i8_buffer(who, "W1", W1, W1_bytes, E * f, d));
    SSG_CHECK(check_i8_buffer(who, "W2", W2, W2_bytes, E * f, d));
    SSG_CHECK(check_i8_buffer(who, "W3", W3, W3_bytes, E * d, f));
    SSG_CHECK(check_ptr(who, "y", y, 16, true));
    SSG_CHECK(check_ptr(who, "workspace", workspace, 256, true));
    const MoeLayout L = moe_layout(*desc);
    if (workspace_bytes < L.total) return fail(SSG_ERR_WORKSPACE, "%s: workspace holds %zu bytes, %zu needed", who, workspace_bytes, L.total);
    SSG_CHECK(check_entry(who));
    uint8_t *b = static_cast<uint8_t *>(workspace);
    hipStream_t st = (hipStream_t)stream;

    ssg::RouteArgs a = route_args(r);
    a.logits = logits; a.bias = bias;
    a.ids = reinterpret_cast<int *>(b + L.ids); a.weights = reinterpret_cast<float *>(b + L.weights);
    a.counts = reinterpret_cast<int *>(b + L.counts); a.offsets = reinterpret_cast<int *>(b + L.offsets);
    a.place = reinterpret_cast<int *>(b + L.place); a.source = reinterpret_cast<int *>(b + L.source);
    a.hist = reinterpret_cast<uint16_t *>(b + L.hist);
    if (few_tokens(*desc)) {
        // h row t k + j for assignment (t, j): no order of dispatch, nothing quantized goes through memory
        a.counts = a.offsets = a.place = a.source = nullptr;
        ssg::launch_route(a, st);
        ssg::I8TokenArgs u;
        u.src = x; u.K = d; u.ld = d; u.bf16 = 1; u.ids = a.ids; u.pairs = r.T * r.k; u.k = r.k;
        u.B = static_cast<const uint8_t *>(W1); u.sb = i8_scales(W1, E * f, d);
        u.B2 = static_cast<const uint8_t *>(W2); u.sb2 = i8_scales(W2, E * f, d);
        u.C = b + L.h; u.N = f; u.ldc = f;
        ssg::launch_i8_token(u, st);
        ssg::I8MixArgs m;
        m.h = b + L.h; m.B = static_cast<const uint8_t *>(W3); m.sb = i8_scales(W3, E * d, f); m.ids = a.ids; m.weights = a.weights;
        m.y = y; m.T = r.T; m.N = d; m.K = f; m.k = r.k; m.y_f32 = desc->y_dtype == SSG_F32; m.o_f32 = f32_results(*desc);
        ssg::launch_i8_mix(m, st);
        return check_launch(who);
    }
    ssg::launch_route(a, st);

    // x in the order of the experts, a scale for each token
    ssg::I8RowsArgs q;
    q.src = x; q.codes = b + L.x_q; q.scales = const_cast<float *>(i8_scales(b + L.x_q, L.rows, d));
    q.rows = L.rows; q.K = d; q.ld = d; q.bf16 = 1; q.source = a.source; q.live_rows = a.offsets + E; q.k = r.k;

    // h = u Swish(g) in bf16, whose error, at most 1/512 of the token's largest value, is half of that of the codes it gets next, 1/254
    ssg::I8GemmArgs g;
    g.A = q.codes; g.sa = q.scales; g.M = L.rows; g.E = (int)E; g.rows_expected = r.T * r.k;
    g.B = static_cast<const uint8_t *>(W1); g.sb = i8_scales(W1, E * f, d);
    g.B2 = static_cast<const uint8_t *>(W2); g.sb2 = i8_scales(W2, E * f, d);
    g.C = b + L.h; g.N = f; g.K = d; g.ldc = f;

    ssg::I8RowsArgs hq;
    hq.src = b + L.h; hq.codes = b + L.h_q; hq.scales = const_cast<float *>(i8_scales(b + L.h_q, L.rows, f));
    hq.rows = L.rows; hq.K = f; hq.ld = f; hq.bf16 = 1; hq.live_rows = a.offsets + E;

    // the experts' results, in fp32 or, where the caller has it so, in y's type: bf16 y is then 2.3e-3 to 3.2e-3 from the sums in 64 bits, and
    // 1.6e-3 to 2.7e-3 from fp32 terms; bf16 terms are half the bytes for the product to write and the sum to read (4096 tokens of 8 rows of
    // 2048 437 us a call for 495, 1041 tokens of 2 rows of 4096 443 for 450, 75 tokens of 8 rows 119 for 122, one token no difference)
    ssg::I8GemmArgs o = g;
    o.A = hq.codes; o.sa = hq.scales; o.B = static_cast<const uint8_t *>(W3); o.sb = i8_scales(W3, E * d, f); o.B2 = nullptr; o.sb2 = nullptr;
    o.C = b + L.o; o.N = d; o.K = f; o.ldc = d; o.c_f32 = f32_results(*desc);

    // the launch that quantizes x lists the row tiles of both products on the side
    int *lists = reinterpret_cast<int *>(b + L.tiles);
    const int up = ssg::i8_row_tiles(g).edge, down = ssg::i8_row_tiles(o).edge;
    q.offsets = a.offsets; q.E = (int)E;
    q.tiles[0].list = lists; q.tiles[0].edge = up;
    if (down != up) { q.tiles[1].list = lists + moe_list_words(L.rows); q.tiles[1].edge = down; }
    g.tiles = lists;
    o.tiles = down != up ? q.tiles[1].list : lists;
    ssg::launch_i8_quantize(q, st);
    ssg::launch_i8_gemm(g, st);
    ssg::launch_i8_quantize(hq, st);
    ssg::launch_i8_gemm(o, st);

    ssg::CombineArgs c;
    c.o = b + L.o; c.y = y; c.place = a.place; c.weights = a.weights; c.T = r.T; c.d = d; c.k = r.k; c.y_f32 = desc->y_dtype == SSG_F32; c.o_f32 = f32_results(*desc);
    ssg::launch_combine(c, st);
    return check_launch(who);
}
