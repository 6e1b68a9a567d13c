// C entry points around the products of experts: routing, the join of their results, activations in 8 bits, root-mean-square norm.
// Argument checks, workspace, launches; everything goes to the context's stream.
#include <math.h>

#include <algorithm>

#include "token_args.h"

using namespace kfac;

namespace {

bool row_sizes_ok(int32_t n, int32_t dim) { return n >= 0 && n <= kMaxPositions && dim >= 1 && dim <= kMaxDim; }
bool rows_ok(const void *p, long long rows, long long cols, long long ld, size_t es) { return p && aligned(p, es) && ld >= cols && spread_ok(rows, ld); }

bool router_ok(const kfac_router *r)
{
    if (!r || r->experts < 1 || r->experts > kMaxRouted || r->fan < 1 || r->fan > kMaxFan) return false;
    if (r->groups < 1 || r->groups > r->experts || r->experts % r->groups || r->top_groups < 1 || r->top_groups > r->groups) return false;
    if (r->group_best < 1 || r->group_best > 2 || (r->scores != KFAC_ROUTE_SOFTMAX && r->scores != KFAC_ROUTE_SIGMOID)) return false;
    if ((r->renormalise != 0 && r->renormalise != 1) || !std::isfinite(r->scale)) return false;
    return r->fan <= r->top_groups * (r->experts / r->groups);
}

RouteArgs route_args(const kfac_router *r, int32_t n, const void *logits, int64_t ld)
{
    RouteArgs a{};
    a.n = n; a.experts = r->experts; a.fan = r->fan; a.groups = r->groups; a.top_groups = r->top_groups;
    a.group_best = r->group_best;
    a.sigmoid = r->scores == KFAC_ROUTE_SIGMOID; a.renormalise = r->renormalise; a.scale = r->scale;
    a.logits = logits; a.ld = ld;
    return a;
}

// What both directions of 8 bits share.
bool bytes_ok(int64_t rows, int32_t cols, const uint8_t *q, int64_t ldq, const uint8_t *scales, int64_t lds)
{
    return rows_ok(q, rows, cols, ldq, 1) && rows_ok(scales, rows, (cols + 31) / 32, lds, 1);
}

}  // namespace

extern "C" {

kfac_status kfac_route(kfac_ctx *ctx, const kfac_router *router, int32_t n, kfac_dtype type, const void *logits, int64_t ld, const float *bias,
                       int32_t *choice, float *gate)
{
    if (!ctx || !router_ok(router) || !type_ok(type) || n < 0 || (long long)n * router->fan > kMaxPositions) return KFAC_ERR_INVALID;
    if (n == 0) return KFAC_OK;
    const long long E = router->experts, choices = (long long)n * router->fan;
    if (!rows_ok(logits, n, E, ld, esize(type)) || !aligned(bias, 4) || !choice || !gate || !aligned(choice, 4) || !aligned(gate, 4)) return KFAC_ERR_INVALID;
    const Range in = matrix(logits, n, E, ld, esize(type)), b = matrix(bias, 1, E, E, 4), c = matrix(choice, 1, choices, choices, 4),
                g = matrix(gate, 1, choices, choices, 4);
    if (overlap(c, g) || overlap(c, in) || overlap(c, b) || overlap(g, in) || overlap(g, b)) return KFAC_ERR_INVALID;
    RouteArgs a = route_args(router, n, logits, ld);
    a.bias = bias; a.choice = choice; a.gate = gate;
    return timed(ctx, KFAC_K_ROUTE, 0, 0.0, (double)n * E * esize(type) + 8.0 * choices, [&] { return launch_route(a, type == KFAC_BF16, ctx_view(ctx).stream); })
               ? KFAC_OK : KFAC_ERR_DEVICE;
}

kfac_status kfac_route_grad(kfac_ctx *ctx, const kfac_router *router, int32_t n, kfac_dtype type, const void *logits, int64_t ld,
                            const int32_t *choice, const float *dgate, void *dlogits, int64_t ldd)
{
    if (!ctx || !router_ok(router) || !type_ok(type) || n < 0 || (long long)n * router->fan > kMaxPositions) return KFAC_ERR_INVALID;
    if (n == 0) return KFAC_OK;
    const long long E = router->experts, choices = (long long)n * router->fan;
    const size_t es = esize(type);
    if (!rows_ok(logits, n, E, ld, es) || !rows_ok(dlogits, n, E, ldd, es) || !choice || !dgate || !aligned(choice, 4) || !aligned(dgate, 4))
        return KFAC_ERR_INVALID;
    const Range out = matrix(dlogits, n, E, ldd, es);
    if (overlap(out, matrix(logits, n, E, ld, es)) || overlap(out, matrix(choice, 1, choices, choices, 4)) || overlap(out, matrix(dgate, 1, choices, choices, 4)))
        return KFAC_ERR_INVALID;
    RouteArgs a = route_args(router, n, logits, ld);
    a.choice = const_cast<int32_t *>(choice); a.dgate = dgate; a.dlogits = dlogits; a.ldd = ldd;   // (the gradient only reads the choices)
    return timed(ctx, KFAC_K_ROUTE, 1, 0.0, 2.0 * n * E * es + 8.0 * choices, [&] { return launch_route_grad(a, type == KFAC_BF16, ctx_view(ctx).stream); })
               ? KFAC_OK : KFAC_ERR_DEVICE;
}

kfac_status kfac_combine(kfac_ctx *ctx, int32_t n, int32_t fan, int32_t dim, kfac_dtype type, const void *y, int64_t ldy, const float *gate,
                         kfac_dtype out_type, const void *residual, int64_t ldr, void *out, int64_t ldo)
{
    if (!ctx || !row_sizes_ok(n, dim) || fan < 1 || n % fan || !type_ok(type) || !type_ok(out_type)) return KFAC_ERR_INVALID;
    if (n == 0) return KFAC_OK;
    const size_t es = esize(type), eo = esize(out_type);
    const int32_t tokens = n / fan;
    if (!rows_ok(y, n, dim, ldy, es) || !rows_ok(out, tokens, dim, ldo, eo) || (residual && !rows_ok(residual, tokens, dim, ldr, eo)) || !aligned(gate, 4))
        return KFAC_ERR_INVALID;
    const Range o = matrix(out, tokens, dim, ldo, eo);
    if (overlap(o, matrix(y, n, dim, ldy, es)) || overlap(o, matrix(gate, 1, n, n, 4))) return KFAC_ERR_INVALID;
    // in place: an element is read and written by the same thread
    if (overlap(o, matrix(residual, tokens, dim, ldr, eo)) && !(out == residual && ldo == ldr)) return KFAC_ERR_INVALID;
    CombineArgs a{};
    a.tokens = tokens; a.fan = fan; a.dim = dim;
    a.y = y; a.ldy = ldy; a.gate = gate; a.r = residual; a.ldr = ldr; a.out = out; a.ldo = ldo;
    return timed(ctx, KFAC_K_COMBINE, 0, 2.0 * n * dim, (double)dim * (es * (double)n + eo * (residual ? 2.0 : 1.0) * tokens),
                 [&] { return launch_combine(a, type == KFAC_BF16, out_type == KFAC_BF16, ctx_view(ctx).stream); }) ? KFAC_OK : KFAC_ERR_DEVICE;
}

kfac_status kfac_combine_grad(kfac_ctx *ctx, int32_t n, int32_t fan, int32_t dim, kfac_dtype type, const void *y, int64_t ldy, const float *gate,
                              kfac_dtype out_type, const void *dout, int64_t ldd, void *dy, int64_t lddy, float *dgate)
{
    if (!ctx || !row_sizes_ok(n, dim) || fan < 1 || n % fan || !type_ok(type) || !type_ok(out_type)) return KFAC_ERR_INVALID;
    if (n == 0) return KFAC_OK;
    if (!dy && !dgate) return KFAC_ERR_INVALID;
    const size_t es = esize(type), eo = esize(out_type);
    const int32_t tokens = n / fan;
    if (!rows_ok(dout, tokens, dim, ldd, eo) || (dgate && (!rows_ok(y, n, dim, ldy, es) || !aligned(dgate, 4))) || (dy && !rows_ok(dy, n, dim, lddy, es)) ||
        !aligned(gate, 4))
        return KFAC_ERR_INVALID;
    const Range rd = matrix(dout, tokens, dim, ldd, eo), ry = dgate ? matrix(y, n, dim, ldy, es) : Range{}, rg = dy ? matrix(gate, 1, n, n, 4) : Range{},
                wy = matrix(dy, n, dim, lddy, es), wg = matrix(dgate, 1, n, n, 4);
    if (overlap(wy, wg) || overlap(wy, rd) || overlap(wy, ry) || overlap(wy, rg) || overlap(wg, rd) || overlap(wg, ry) || overlap(wg, rg))
        return KFAC_ERR_INVALID;
    CombineArgs a{};
    a.tokens = tokens; a.fan = fan; a.dim = dim;
    a.y = y; a.ldy = ldy; a.gate = gate; a.dout = dout; a.ldd = ldd; a.dy = dy; a.lddy = lddy; a.dgate = dgate;
    return timed(ctx, KFAC_K_COMBINE, 1, 3.0 * n * dim, (double)dim * (es * (double)n * ((dgate != nullptr) + (dy != nullptr)) + eo * (double)tokens),
                 [&] { return launch_combine_grad(a, type == KFAC_BF16, out_type == KFAC_BF16, ctx_view(ctx).stream); }) ? KFAC_OK : KFAC_ERR_DEVICE;
}

kfac_status kfac_keep(kfac_ctx *ctx, int64_t rows, int32_t cols, kfac_dtype type, const void *x, int64_t ldx, uint8_t *q, int64_t ldq,
                      uint8_t *scales, int64_t lds)
{
    if (!ctx || !type_ok(type) || rows < 0 || rows > ((int64_t)1 << 40) || cols < 0 || cols > kMaxPositions) return KFAC_ERR_INVALID;
    if (rows == 0 || cols == 0) return KFAC_OK;
    if (!rows_ok(x, rows, cols, ldx, esize(type)) || !bytes_ok(rows, cols, q, ldq, scales, lds)) return KFAC_ERR_INVALID;
    const Range in = matrix(x, rows, cols, ldx, esize(type)), o = matrix(q, rows, cols, ldq, 1), e = matrix(scales, rows, (cols + 31) / 32, lds, 1);
    if (overlap(o, e) || overlap(o, in) || overlap(e, in)) return KFAC_ERR_INVALID;
    KeepArgs a{};
    a.rows = rows; a.cols = cols; a.x = x; a.ldx = ldx; a.q = q; a.ldq = ldq; a.scales = scales; a.lds = lds;
    return timed(ctx, KFAC_K_KEEP, 0, 0.0, (double)rows * cols * (esize(type) + 1 + 1.0 / 32), [&] { return launch_keep(a, type == KFAC_BF16, ctx_view(ctx).stream); })
               ? KFAC_OK : KFAC_ERR_DEVICE;
}

kfac_status kfac_restore(kfac_ctx *ctx, int64_t rows, int32_t cols, const uint8_t *q, int64_t ldq, const uint8_t *scales, int64_t lds,
                         kfac_dtype type, void *x, int64_t ldx)
{
    if (!ctx || !type_ok(type) || rows < 0 || rows > ((int64_t)1 << 40) || cols < 0 || cols > kMaxPositions) return KFAC_ERR_INVALID;
    if (rows == 0 || cols == 0) return KFAC_OK;
    if (!rows_ok(x, rows, cols, ldx, esize(type)) || !bytes_ok(rows, cols, q, ldq, scales, lds)) return KFAC_ERR_INVALID;
    const Range out = matrix(x, rows, cols, ldx, esize(type));
    if (overlap(out, matrix(q, rows, cols, ldq, 1)) || overlap(out, matrix(scales, rows, (cols + 31) / 32, lds, 1))) return KFAC_ERR_INVALID;
    KeepArgs a{};
    a.rows = rows; a.cols = cols; a.back = x; a.ldx = ldx; a.ldq = ldq; a.lds = lds;
    a.q = const_cast<uint8_t *>(q); a.scales = const_cast<uint8_t *>(scales);   // (only read in this direction)
    return timed(ctx, KFAC_K_KEEP, 1, 0.0, (double)rows * cols * (esize(type) + 1 + 1.0 / 32), [&] { return launch_restore(a, type == KFAC_BF16, ctx_view(ctx).stream); })
               ? KFAC_OK : KFAC_ERR_DEVICE;
}

kfac_status kfac_rms_norm(kfac_ctx *ctx, int32_t n, int32_t dim, kfac_dtype type, const void *x, int64_t ldx, kfac_dtype stream_type,
                          const void *residual, int64_t ldr, void *h, int64_t ldh, const float *gamma, float eps, void *y, int64_t ldy,
                          uint8_t *q, int64_t ldq, uint8_t *scales, int64_t lds)
{
    if (!ctx || n < 0 || n > kMaxPositions || dim < 1 || dim > kMaxNorm || !type_ok(type) || !type_ok(stream_type)) return KFAC_ERR_INVALID;
    if (!std::isfinite(eps) || eps < 0.f) return KFAC_ERR_INVALID;
    if (n == 0) return KFAC_OK;
    if ((!residual) != (!h) || (!residual && stream_type != type) || (!y && !q) || (!q) != (!scales)) return KFAC_ERR_INVALID;
    const size_t es = esize(type), et = esize(stream_type);
    if (!rows_ok(x, n, dim, ldx, es) || !gamma || !aligned(gamma, 4) || (residual && (!rows_ok(residual, n, dim, ldr, et) || !rows_ok(h, n, dim, ldh, et))) ||
        (y && !rows_ok(y, n, dim, ldy, es)) || (q && !bytes_ok(n, dim, q, ldq, scales, lds)))
        return KFAC_ERR_INVALID;
    const Range rx = matrix(x, n, dim, ldx, es), rr = matrix(residual, n, dim, ldr, et), rg = matrix(gamma, 1, dim, dim, 4), wh = matrix(h, n, dim, ldh, et),
                wy = matrix(y, n, dim, ldy, es), wq = matrix(q, n, dim, ldq, 1), ws = matrix(scales, n, (dim + 31) / 32, lds, 1);
    // in place: a row is read before it is written, by the same threads
    if (overlap(wh, rx) && !(h == x && ldh == ldx && type == stream_type)) return KFAC_ERR_INVALID;
    if (overlap(wh, rr) && !(h == residual && ldh == ldr)) return KFAC_ERR_INVALID;
    if (overlap(wy, rx) && !(y == x && ldy == ldx)) return KFAC_ERR_INVALID;
    if (overlap(wy, rr) || overlap(wh, wy) || overlap(wh, rg) || overlap(wy, rg) || overlap(wq, ws)) return KFAC_ERR_INVALID;
    for (const Range &w : {wq, ws})
        if (overlap(w, rx) || overlap(w, rr) || overlap(w, rg) || overlap(w, wh) || overlap(w, wy)) return KFAC_ERR_INVALID;
    NormArgs a{};
    a.n = n; a.dim = dim; a.x = x; a.ldx = ldx; a.r = residual; a.ldr = ldr; a.h = h; a.ldh = ldh; a.gamma = gamma; a.eps = eps;
    a.y = y; a.ldy = ldy; a.q = q; a.ldq = ldq; a.scales = scales; a.lds = lds;
    return timed(ctx, KFAC_K_NORM, 0, 4.0 * n * dim, (double)n * dim * (es * (1.0 + (y != nullptr)) + (residual ? 2.0 * et : 0.0) + (q ? 1.0 + 1.0 / 32 : 0.0)),
                 [&] { return launch_norm(a, type == KFAC_BF16, stream_type == KFAC_BF16, ctx_view(ctx).stream); }) ? KFAC_OK : KFAC_ERR_DEVICE;
}

size_t kfac_rms_norm_workspace_bytes(int32_t n, int32_t dim)
{
    if (n < 0 || n > kMaxPositions || dim < 1 || dim > kMaxNorm) return 0;
    return std::max<size_t>(256, ((size_t)norm_parts(n, dim) * 2 * dim * sizeof(float) + 255) / 256 * 256);
}

kfac_status kfac_rms_norm_grad(kfac_ctx *ctx, int32_t n, int32_t dim, kfac_dtype type, const void *dy, int64_t lddy, kfac_dtype stream_type,
                               const void *h, int64_t ldh, const float *gamma, float eps, const void *dstream, int64_t ldr, void *dh,
                               int64_t lddh, float *dgamma, float decay, float *F_ema)
{
    if (!ctx || n < 0 || n > kMaxPositions || dim < 1 || dim > kMaxNorm || !type_ok(type) || !type_ok(stream_type)) return KFAC_ERR_INVALID;
    if (!std::isfinite(eps) || eps < 0.f || !(decay >= 0.f && decay < 1.f) || !aligned(dgamma, 4) || !aligned(F_ema, 4)) return KFAC_ERR_INVALID;
    if (!dh && !dgamma && !F_ema) return n == 0 ? KFAC_OK : KFAC_ERR_INVALID;
    const size_t es = esize(type), et = esize(stream_type);
    if (n > 0 && (!rows_ok(dy, n, dim, lddy, es) || !rows_ok(h, n, dim, ldh, et) || !gamma || !aligned(gamma, 4) ||
                  (dstream && !rows_ok(dstream, n, dim, ldr, et)) || (dh && !rows_ok(dh, n, dim, lddh, et))))
        return KFAC_ERR_INVALID;
    const Range ry = matrix(dy, n, dim, lddy, es), rh = matrix(h, n, dim, ldh, et), rr = dh ? matrix(dstream, n, dim, ldr, et) : Range{},
                rg = matrix(gamma, 1, dim, dim, 4), wh = matrix(dh, n, dim, lddh, et), wg = matrix(dgamma, 1, dim, dim, 4), wf = matrix(F_ema, 1, dim, dim, 4);
    if (overlap(wh, rr) && !(dh == dstream && lddh == ldr)) return KFAC_ERR_INVALID;
    if (overlap(wh, ry) && !(dh == dy && lddh == lddy && type == stream_type)) return KFAC_ERR_INVALID;
    if (overlap(wh, rh) || overlap(wh, rg) || overlap(wg, wf)) return KFAC_ERR_INVALID;
    for (const Range &w : {wg, wf})
        if (overlap(w, ry) || overlap(w, rh) || overlap(w, rr) || overlap(w, rg) || overlap(w, wh)) return KFAC_ERR_INVALID;
    const CtxView c = ctx_view(ctx);
    const bool columns = dgamma || F_ema;
    if (columns && kfac_rms_norm_workspace_bytes(n, dim) > c.ws_bytes) return KFAC_ERR_WORKSPACE;
    if (n == 0 && !columns) return KFAC_OK;   // no rows, no sums
    NormGradArgs a{};
    a.n = n; a.dim = dim; a.dy = dy; a.lddy = lddy; a.h = h; a.ldh = ldh; a.r = dstream; a.ldr = ldr; a.dh = dh; a.lddh = lddh;
    a.gamma = gamma; a.eps = eps; a.dgamma = dgamma; a.F = F_ema; a.decay = decay; a.partial = (float *)c.ws;
    const double e = (double)n * dim;
    // (no rows: nothing to read, gamma neither; the sums of columns are zeros)
    bool ok = n == 0 || timed(ctx, KFAC_K_NORM, 1, 12.0 * e, e * (es + et * (1.0 + (dh ? 1.0 + (dstream != nullptr) : 0.0))),
                              [&] { return launch_norm_grad(a, type == KFAC_BF16, stream_type == KFAC_BF16, c.stream); });
    if (columns) ok = ok && timed(ctx, KFAC_K_NORM, 2, 0.0, 8.0 * norm_parts(n, dim) * dim, [&] { return launch_norm_join(a, c.stream); });
    return ok ? KFAC_OK : KFAC_ERR_DEVICE;
}

}  // extern "C"
