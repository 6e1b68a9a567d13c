// C entry points of the token and expert layers: segments, embedding, dropout, products grouped by expert and their factors.
// Argument checks, workspace, launches; no tables and no internal streams: everything goes to the context's stream.
#include <math.h>

#include <algorithm>

#include "token_args.h"

using namespace kfac;

namespace {

bool segments_ok(int32_t n, int32_t num) { return n >= 0 && n <= kMaxPositions && num >= 1 && num < (1 << 30); }

size_t embedding_grad_scratch(char *base, int n, int vocab, int dim, SegmentScratch *seg, int **pos, float **partial)
{
    size_t used = segment_scratch(base, n, vocab, seg);
    auto take = [&](size_t bytes) {
        char *p = base ? base + used : nullptr;
        used += (bytes + 255) / 256 * 256;
        return p;
    };
    char *order = take(sizeof(int) * (size_t)std::max(n, 1));
    char *part = take(2 * (size_t)embedding_most_chunks(n) * (size_t)dim * sizeof(float));
    if (pos) *pos = (int *)order;
    if (partial) *partial = (float *)part;
    return used;
}

// Experts that the calls take.
bool experts_ok(const kfac_layer *L, int32_t experts, int32_t n)
{
    if (!L || kfac_layer_dims(L, nullptr, nullptr, nullptr, nullptr) != KFAC_OK) return false;
    if (L->k != 1 || L->stride != 1 || L->pad != 0 || L->h_in != 1 || L->w_in != 1) return false;
    if (experts < 1 || experts > kMaxExperts || n < 0 || n > kMaxPositions) return false;
    // tiles of one launch, 64 x 64 elements at least
    const long long ti = (L->c_in + 63) / 64, to = (L->c_out + 63) / 64;
    if (((long long)n / 64 + experts + 1) * std::max(ti, to) >= (1LL << 30)) return false;
    return experts * (ti * to + ti * (ti + 1) / 2 + to * (to + 1) / 2 + 16) < (1LL << 30);
}

// What the four expert calls share.
bool expert_ok(const kfac_ctx *ctx, const kfac_layer *L, int32_t experts, int32_t n, int32_t fan, kfac_dtype type, const int32_t *offsets)
{
    return ctx && offsets && aligned(offsets, 4) && type_ok(type) && experts_ok(L, experts, n) && fan >= 1 && n % fan == 0;
}

ExpertArgs expert_args(const kfac_layer *L, int32_t experts, int32_t n, int32_t fan, const int32_t *order, const int32_t *offsets)
{
    ExpertArgs a{};
    a.order = order; a.offsets = offsets;
    a.n = n; a.experts = experts; a.fan = fan;
    a.ci = L->c_in; a.co = L->c_out; a.bias = L->bias;
    return a;
}

bool run_expert(kfac_ctx *ctx, ExpertOp op, const ExpertArgs &a, kfac_dtype type, double flops, double bytes)
{
    const CtxView c = ctx_view(ctx);
    return timed(ctx, KFAC_K_EXPERT, (int)op, flops, bytes, [&] {
        return (a.partial ? launch_expert_pieces : launch_expert)(op, a, type == KFAC_BF16, c.fp32_planes, c.stream);
    });
}

// The checks of kfac_expert_grad_weight and kfac_stats_expert, and what they launch.  in: what x is read from, one or two tensors.
struct Inputs { Range a, b; };
Inputs plain_inputs(const kfac_layer *L, int32_t n, int32_t fan, kfac_dtype type, const void *x, int64_t ldx)
{
    return L && fan >= 1 && n > 0 && ldx >= L->c_in && ldx <= kMaxPositions ? Inputs{matrix(x, n / fan, L->c_in, ldx, esize(type)), Range{}} : Inputs{};
}
Inputs kept_inputs(const kfac_layer *L, int32_t n, int32_t fan, const uint8_t *q, int64_t ldq, const uint8_t *scales, int64_t lds)
{
    return {matrix(q, n / fan, L->c_in, ldq, 1), matrix(scales, n / fan, (L->c_in + 31) / 32, lds, 1)};
}
kfac_status weight_args(kfac_ctx *ctx, const kfac_layer *L, int32_t experts, int32_t n, int32_t fan, kfac_dtype type, const int32_t *order,
                        const int32_t *offsets, const Inputs &in, const void *x, int64_t ldx, const void *dy, int64_t ldy, float *dW, ExpertArgs &a)
{
    if (!expert_ok(ctx, L, experts, n, fan, type, offsets) || !aligned(order, 4) || !dW || !aligned(dW, 4)) return KFAC_ERR_INVALID;
    if (ldx < L->c_in || ldy < L->c_out || ldx > kMaxPositions || ldy > kMaxPositions) return KFAC_ERR_INVALID;
    const size_t es = esize(type);
    if (n > 0 && (!x || !dy || !aligned(x, es) || !aligned(dy, es))) return KFAC_ERR_INVALID;
    const Range out = matrix(dW, (long long)experts * L->c_out, L->c_in + L->bias, L->c_in + L->bias, 4);
    if (overlap(out, in.a) || overlap(out, in.b) || overlap(out, matrix(dy, n, L->c_out, ldy, es))) return KFAC_ERR_INVALID;
    a = expert_args(L, experts, n, fan, order, offsets);
    a.x = x; a.ldx = ldx; a.dy = dy; a.ldy = ldy; a.dW = dW;
    return KFAC_OK;
}
kfac_status run_weight(kfac_ctx *ctx, const ExpertArgs &a, kfac_dtype type)
{
    return run_expert(ctx, EXPERT_GRAD_WEIGHT, a, type, 2.0 * a.n * a.ci * a.co,
                      esize(type) * (double)a.n * (a.ci / (double)a.fan + a.co) + 4.0 * a.experts * a.co * (a.ci + a.bias)) ? KFAC_OK : KFAC_ERR_DEVICE;
}

kfac_status stats_args(kfac_ctx *ctx, const kfac_layer *L, int32_t experts, int32_t n, int32_t fan, kfac_dtype in, const int32_t *order,
                       const int32_t *offsets, const Inputs &from, const void *x, int64_t ldx, const void *grad_out, int64_t ldg, float decay,
                       float *A_ema, float *G_ema, ExpertArgs &a)
{
    if (!expert_ok(ctx, L, experts, n, fan, in, offsets) || !aligned(order, 4)) return KFAC_ERR_INVALID;
    if (!(decay >= 0.f && decay < 1.f) || (!A_ema && !G_ema) || !aligned(A_ema, 4) || !aligned(G_ema, 4)) return KFAC_ERR_INVALID;
    const size_t es = esize(in);
    if (A_ema && (ldx < L->c_in || ldx > kMaxPositions || (n > 0 && (!x || !aligned(x, es))))) return KFAC_ERR_INVALID;
    if (G_ema && (ldg < L->c_out || ldg > kMaxPositions || (n > 0 && (!grad_out || !aligned(grad_out, es))))) return KFAC_ERR_INVALID;
    const long long dA = L->c_in + L->bias, dG = L->c_out;
    const Range rg = G_ema ? matrix(grad_out, n, L->c_out, ldg, es) : Range{}, A = matrix(A_ema, experts * dA, dA, dA, 4),
                G = matrix(G_ema, experts * dG, dG, dG, 4);
    if (overlap(A, G) || overlap(A, rg) || overlap(G, rg)) return KFAC_ERR_INVALID;
    if (A_ema && (overlap(A, from.a) || overlap(A, from.b) || overlap(G, from.a) || overlap(G, from.b))) return KFAC_ERR_INVALID;
    a = expert_args(L, experts, n, fan, order, offsets);
    a.x = x; a.ldx = ldx; a.dy = grad_out; a.ldy = ldg;
    a.A = A_ema; a.G = G_ema; a.decay = decay;
    return KFAC_OK;
}
kfac_status run_stats(kfac_ctx *ctx, const ExpertArgs &a, kfac_dtype in)
{
    const double dA = a.ci + a.bias, dG = a.co, fa = a.A ? dA * dA : 0.0, fg = a.G ? dG * dG : 0.0, es = esize(in);
    const double read = (a.A ? es * a.n / a.fan * a.ci : 0.0) + (a.G ? es * a.n * a.co : 0.0);
    return run_expert(ctx, EXPERT_STATS, a, in, a.n * (fa + fg), read + 4.0 * a.experts * (fa + fg)) ? KFAC_OK : KFAC_ERR_DEVICE;
}

// Inputs of experts that were kept in 8 bits; in the workspace as values, rows a whole number of 16-byte chunks apart: sorted by place for up to
// kPieceExperts experts (the products then cut long experts into pieces, whose sums follow), by token for more.
int64_t kept_row(const kfac_layer *L) { return ((int64_t)L->c_in + 63) / 64 * 64; }
size_t kept_bytes(const kfac_layer *L, int32_t experts, int32_t n, int32_t fan, kfac_dtype type)
{
    return ((size_t)(experts <= kPieceExperts ? n : n / fan) * kept_row(L) * esize(type) + 255) / 256 * 256;
}
size_t kept_scratch(const kfac_layer *L, int32_t experts, int32_t n, int32_t fan, kfac_dtype type)
{
    return kept_bytes(L, experts, n, fan, type) + (experts <= kPieceExperts ? expert_pieces_bytes(experts, n, L->c_in, L->c_out) : 0);
}
bool kept_ok(const kfac_layer *L, int32_t n, int32_t fan, const uint8_t *q, int64_t ldq, const uint8_t *scales, int64_t lds)
{
    return ldq >= L->c_in && lds >= (L->c_in + 31) / 32 && ldq <= kMaxPositions && lds <= kMaxPositions && (n == 0 || (q && scales));
}
// Brings them there and sends the product after them.
kfac_status run_kept(kfac_ctx *ctx, ExpertOp op, ExpertArgs a, const kfac_layer *L, kfac_dtype type, const uint8_t *q, int64_t ldq, const uint8_t *scales,
                     int64_t lds)
{
    const CtxView c = ctx_view(ctx);
    KeepArgs k{};
    const bool pieces = a.experts <= kPieceExperts;
    k.gather = pieces; k.order = a.order; k.fan = a.fan;
    k.rows = pieces ? a.n : a.n / a.fan; k.cols = L->c_in; k.back = c.ws; k.ldx = kept_row(L);
    k.q = const_cast<uint8_t *>(q); k.ldq = ldq; k.scales = const_cast<uint8_t *>(scales); k.lds = lds;   // (only read)
    if (k.rows > 0 && !timed(ctx, KFAC_K_KEEP, 1, 0.0, (double)k.rows * k.cols * (esize(type) + 1 + 1.0 / 32),
                             [&] { return launch_restore(k, type == KFAC_BF16, c.stream); })) return KFAC_ERR_DEVICE;
    if (pieces) a.partial = (float *)(c.ws + kept_bytes(L, a.experts, a.n, a.fan, type));
    return op == EXPERT_GRAD_WEIGHT ? run_weight(ctx, a, type) : run_stats(ctx, a, type);
}

}  // namespace

extern "C" {

size_t kfac_segments_workspace_bytes(int32_t n, int32_t num)
{
    return segments_ok(n, num) ? segment_scratch(nullptr, n, num, nullptr) : 0;
}

kfac_status kfac_segments(kfac_ctx *ctx, int32_t n, const void *ids, int32_t id_bits, int32_t num, int32_t *order, int32_t *offsets)
{
    if (!ctx || !segments_ok(n, num) || (id_bits != 32 && id_bits != 64) || !offsets || (n > 0 && (!ids || !order))) return KFAC_ERR_INVALID;
    if (!aligned(ids, id_bits / 8) || !aligned(order, 4) || !aligned(offsets, 4)) return KFAC_ERR_INVALID;
    const Range in{(const char *)ids, (size_t)n * (id_bits / 8)}, o{(const char *)order, 4 * (size_t)n}, f{(const char *)offsets, 4 * ((size_t)num + 1)};
    if (overlap(in, o) || overlap(in, f) || overlap(o, f)) return KFAC_ERR_INVALID;
    const CtxView c = ctx_view(ctx);
    SegmentScratch w;
    if (segment_scratch(c.ws, n, num, &w) > c.ws_bytes) return KFAC_ERR_WORKSPACE;
    return timed(ctx, KFAC_K_SEGMENTS, 0, 0.0, (double)in.size + o.size + f.size,
                 [&] { return launch_segments(ids, id_bits, n, num, w, order, nullptr, offsets, nullptr, c.stream); }) ? KFAC_OK : KFAC_ERR_DEVICE;
}

kfac_status kfac_embedding(kfac_ctx *ctx, int32_t n, const void *ids, int32_t id_bits, int32_t vocab, int32_t dim, kfac_dtype table_type,
                           const void *table, int64_t ld_table, float scale, kfac_dtype out_type, void *out, int64_t ld_out)
{
    if (!ctx || !segments_ok(n, vocab) || dim < 1 || dim > kMaxDim || (id_bits != 32 && id_bits != 64)) return KFAC_ERR_INVALID;
    if (!type_ok(table_type) || !type_ok(out_type) || !std::isfinite(scale)) return KFAC_ERR_INVALID;
    if (ld_table < dim || ld_out < dim || !spread_ok(vocab, ld_table) || !spread_ok(n, ld_out)) return KFAC_ERR_INVALID;
    if (n == 0) return KFAC_OK;
    if (!ids || !table || !out || !aligned(ids, id_bits / 8) || !aligned(table, esize(table_type)) || !aligned(out, esize(out_type))) return KFAC_ERR_INVALID;
    const Range o = matrix(out, n, dim, ld_out, esize(out_type));
    if (overlap(o, matrix(table, vocab, dim, ld_table, esize(table_type))) || overlap(o, Range{ids, (size_t)n * (id_bits / 8)}))
        return KFAC_ERR_INVALID;
    return timed(ctx, KFAC_K_EMBEDDING, 0, (double)n * dim, (double)n * dim * (esize(table_type) + esize(out_type)), [&] {
        return launch_embedding(ids, id_bits, n, vocab, dim, table_type == KFAC_BF16, table, ld_table, scale, out_type == KFAC_BF16, out, ld_out,
                                ctx_view(ctx).stream);
    }) ? KFAC_OK : KFAC_ERR_DEVICE;
}

size_t kfac_embedding_workspace_bytes(int32_t n, int32_t vocab, int32_t dim)
{
    if (!segments_ok(n, vocab) || dim < 1 || dim > kMaxDim) return 0;
    return embedding_grad_scratch(nullptr, n, vocab, dim, nullptr, nullptr, nullptr);
}

kfac_status kfac_embedding_grad(kfac_ctx *ctx, int32_t n, const void *ids, int32_t id_bits, int32_t vocab, int32_t dim, kfac_dtype type,
                                const void *grad_out, int64_t ld_grad, float scale, int32_t accumulate, float *dW, float decay, float *A_diag)
{
    if (!ctx || !segments_ok(n, vocab) || dim < 1 || dim > kMaxDim || (id_bits != 32 && id_bits != 64) || !type_ok(type)) return KFAC_ERR_INVALID;
    if (!std::isfinite(scale) || !(decay >= 0.f && decay < 1.f) || ld_grad < dim || !spread_ok(n, ld_grad) || !dW) return KFAC_ERR_INVALID;
    if (!aligned(dW, 4) || !aligned(A_diag, 4) || (n > 0 && (!ids || !grad_out || !aligned(ids, id_bits / 8) || !aligned(grad_out, esize(type)))))
        return KFAC_ERR_INVALID;
    if (((long long)n / embedding_chunk(n) + 1) * (dim / 256 + 1) >= (1LL << 30)) return KFAC_ERR_INVALID;   // workgroups of one launch
    const Range w = matrix(dW, vocab, dim, dim, 4), d = matrix(A_diag, 1, vocab, vocab, 4), g = matrix(grad_out, n, dim, ld_grad, esize(type)),
                in{(const char *)ids, (size_t)n * (id_bits / 8)};
    if (overlap(w, d) || overlap(w, g) || overlap(w, in) || overlap(d, g) || overlap(d, in)) return KFAC_ERR_INVALID;
    const CtxView c = ctx_view(ctx);
    SegmentScratch seg;
    EmbeddingGrad a{};
    int *pos;
    if (embedding_grad_scratch(c.ws, n, vocab, dim, &seg, &pos, &a.partial) > c.ws_bytes) return KFAC_ERR_WORKSPACE;
    a.pos = pos; a.keys = seg.keys[0];
    a.n = n; a.vocab = vocab; a.dim = dim;
    a.g = grad_out; a.ld = ld_grad; a.bf16 = type == KFAC_BF16;
    a.accumulate = accumulate != 0;
    a.scale = scale; a.share = n > 0 ? (1.f - decay) / (float)n : 0.f;
    a.dW = dW; a.A = A_diag;
    a.chunk = embedding_chunk(n);
    Fill fill{};
    if (!accumulate) { fill.data = dW; fill.count = (long long)vocab * dim; }
    if (A_diag && n > 0) { fill.decayed = A_diag; fill.n_decayed = vocab; fill.decay = decay; }   // no positions: no mean to add
    const double moved = (double)n * dim * esize(type), written = 4.0 * vocab * dim;
    bool ok;
    if (n > 0) {
        const int *keys = nullptr;
        ok = timed(ctx, KFAC_K_SEGMENTS, 0, 0.0, 2.0 * in.size + written, [&] { return launch_segments(ids, id_bits, n, vocab, seg, pos, &keys, nullptr, &fill, c.stream); });
        a.keys = keys;
        ok = ok && timed(ctx, KFAC_K_EMBEDDING, 1, (double)n * dim, moved, [&] { return launch_embedding_sum(a, c.stream); });
        ok = ok && timed(ctx, KFAC_K_EMBEDDING, 2, 0.0, 0.0, [&] { return launch_embedding_join(a, c.stream); });
    } else {
        ok = timed(ctx, KFAC_K_SEGMENTS, 0, 0.0, written, [&] { return launch_fill(fill, c.stream); });
    }
    return ok ? KFAC_OK : KFAC_ERR_DEVICE;
}

kfac_status kfac_dropout(kfac_ctx *ctx, int64_t rows, int64_t cols, kfac_dtype type, const void *x, int64_t ldx, const void *residual, int64_t ldr,
                         float p, uint64_t seed, uint64_t offset, void *y, int64_t ldy)
{
    constexpr int64_t most = (int64_t)1 << 40;
    if (!ctx || !type_ok(type) || rows < 0 || cols < 0 || rows > most || cols > most || !(p >= 0.f && p <= 1.f)) return KFAC_ERR_INVALID;
    if (rows == 0 || cols == 0) return KFAC_OK;
    if (rows > most / cols || ldx < cols || ldy < cols || (residual && ldr < cols) || ldr > most) return KFAC_ERR_INVALID;
    if (!spread_ok(rows, ldx) || !spread_ok(rows, ldy) || (residual && !spread_ok(rows, ldr))) return KFAC_ERR_INVALID;
    if (rows > 1 && cols > ((int64_t)1 << 32)) return KFAC_ERR_INVALID;
    if (!x || !y || !aligned(x, esize(type)) || !aligned(y, esize(type)) || !aligned(residual, esize(type))) return KFAC_ERR_INVALID;
    const Range out = matrix(y, rows, cols, ldy, esize(type)), in = matrix(x, rows, cols, ldx, esize(type)),
                res = matrix(residual, rows, cols, ldr, esize(type));
    // in place: an element is read and written by the same thread
    if (overlap(out, in) && !(y == x && ldy == ldx)) return KFAC_ERR_INVALID;
    if (overlap(out, res) && !(y == residual && ldy == ldr)) return KFAC_ERR_INVALID;
    DropoutArgs a{};
    a.rows = rows; a.cols = cols;
    a.x = x; a.r = residual; a.y = y;
    a.ldx = ldx; a.ldr = ldr; a.ldy = ldy;
    a.threshold = (unsigned)lrint((double)p * 65536.0);
    a.factor = a.threshold < 65536u ? (float)(65536.0 / (65536.0 - a.threshold)) : 0.f;
    a.seed = seed; a.offset = offset;
    const double e = (double)rows * cols;
    return timed(ctx, KFAC_K_DROPOUT, 0, 0.0, e * esize(type) * (residual ? 3 : 2),
                 [&] { return launch_dropout(a, type == KFAC_BF16, ctx_view(ctx).stream); }) ? KFAC_OK : KFAC_ERR_DEVICE;
}

size_t kfac_expert_workspace_bytes(const kfac_layer *L, int32_t experts, int32_t n)
{
    return experts_ok(L, experts, n) ? 256 : 0;   // (they use none; 0 is for what they refuse)
}

kfac_status kfac_expert_forward(kfac_ctx *ctx, const kfac_layer *L, int32_t experts, int32_t n, int32_t fan, kfac_dtype type, const int32_t *order,
                                const int32_t *offsets, const void *x, int64_t ldx, const void *W, int64_t ldw, void *y, int64_t ldy)
{
    if (!expert_ok(ctx, L, experts, n, fan, type, offsets) || !aligned(order, 4)) return KFAC_ERR_INVALID;
    if (ldx < L->c_in || ldy < L->c_out || ldw < L->c_in + L->bias || ldx > kMaxPositions || ldy > kMaxPositions || ldw > kMaxPositions) return KFAC_ERR_INVALID;
    if (n == 0) return KFAC_OK;
    const size_t es = esize(type);
    if (!x || !W || !y || !aligned(x, es) || !aligned(W, es) || !aligned(y, es)) return KFAC_ERR_INVALID;
    const Range out = matrix(y, n, L->c_out, ldy, es);
    if (overlap(out, matrix(x, n / fan, L->c_in, ldx, es)) || overlap(out, matrix(W, (long long)experts * L->c_out, L->c_in + L->bias, ldw, es)))
        return KFAC_ERR_INVALID;
    ExpertArgs a = expert_args(L, experts, n, fan, order, offsets);
    a.x = x; a.ldx = ldx; a.W = W; a.ldw = ldw; a.out = y; a.ldo = ldy;
    return run_expert(ctx, EXPERT_FORWARD, a, type, 2.0 * n * L->c_in * L->c_out,
                      es * ((double)n * (L->c_in / (double)fan + L->c_out) + (double)experts * L->c_in * L->c_out)) ? KFAC_OK : KFAC_ERR_DEVICE;
}

kfac_status kfac_expert_grad_input(kfac_ctx *ctx, const kfac_layer *L, int32_t experts, int32_t n, kfac_dtype type, const int32_t *order,
                                   const int32_t *offsets, const void *dy, int64_t ldy, const void *W, int64_t ldw, void *dx, int64_t ldx)
{
    if (!expert_ok(ctx, L, experts, n, 1, type, offsets) || !aligned(order, 4)) return KFAC_ERR_INVALID;
    if (ldx < L->c_in || ldy < L->c_out || ldw < L->c_in + L->bias || ldx > kMaxPositions || ldy > kMaxPositions || ldw > kMaxPositions) return KFAC_ERR_INVALID;
    if (n == 0) return KFAC_OK;
    const size_t es = esize(type);
    if (!dy || !W || !dx || !aligned(dy, es) || !aligned(W, es) || !aligned(dx, es)) return KFAC_ERR_INVALID;
    const Range out = matrix(dx, n, L->c_in, ldx, es);
    if (overlap(out, matrix(dy, n, L->c_out, ldy, es)) || overlap(out, matrix(W, (long long)experts * L->c_out, L->c_in + L->bias, ldw, es)))
        return KFAC_ERR_INVALID;
    ExpertArgs a = expert_args(L, experts, n, 1, order, offsets);
    a.dy = dy; a.ldy = ldy; a.W = W; a.ldw = ldw; a.out = dx; a.ldo = ldx;
    return run_expert(ctx, EXPERT_GRAD_INPUT, a, type, 2.0 * n * L->c_in * L->c_out,
                      es * ((double)n * (L->c_in + L->c_out) + (double)experts * L->c_in * L->c_out)) ? KFAC_OK : KFAC_ERR_DEVICE;
}

kfac_status kfac_expert_grad_weight(kfac_ctx *ctx, const kfac_layer *L, int32_t experts, int32_t n, int32_t fan, kfac_dtype type, const int32_t *order,
                                    const int32_t *offsets, const void *x, int64_t ldx, const void *dy, int64_t ldy, float *dW)
{
    ExpertArgs a;
    const kfac_status st = weight_args(ctx, L, experts, n, fan, type, order, offsets, plain_inputs(L, n, fan, type, x, ldx), x, ldx, dy, ldy, dW, a);
    return st == KFAC_OK ? run_weight(ctx, a, type) : st;
}

kfac_status kfac_stats_expert(kfac_ctx *ctx, const kfac_layer *L, int32_t experts, int32_t n, int32_t fan, kfac_dtype in, const int32_t *order,
                              const int32_t *offsets, const void *x, int64_t ldx, const void *grad_out, int64_t ldg, float decay, float *A_ema,
                              float *G_ema)
{
    ExpertArgs a;
    const kfac_status st = stats_args(ctx, L, experts, n, fan, in, order, offsets, plain_inputs(L, n, fan, in, x, ldx), x, ldx, grad_out, ldg, decay,
                                      A_ema, G_ema, a);
    return st == KFAC_OK && n > 0 ? run_stats(ctx, a, in) : st;   // (n = 0: no expert has rows)
}

size_t kfac_kept_workspace_bytes(const kfac_layer *L, int32_t experts, int32_t n, int32_t fan)
{
    return experts_ok(L, experts, n) && fan >= 1 && n % fan == 0 ? std::max<size_t>(256, kept_scratch(L, experts, n, fan, KFAC_F32)) : 0;
}

kfac_status kfac_expert_grad_weight_kept(kfac_ctx *ctx, const kfac_layer *L, int32_t experts, int32_t n, int32_t fan, kfac_dtype type,
                                         const int32_t *order, const int32_t *offsets, const uint8_t *q, int64_t ldq, const uint8_t *scales,
                                         int64_t lds, const void *dy, int64_t ldy, float *dW)
{
    if (!expert_ok(ctx, L, experts, n, fan, type, offsets) || !kept_ok(L, n, fan, q, ldq, scales, lds)) return KFAC_ERR_INVALID;
    const CtxView c = ctx_view(ctx);
    ExpertArgs a;
    const kfac_status st = weight_args(ctx, L, experts, n, fan, type, order, offsets, kept_inputs(L, n, fan, q, ldq, scales, lds), c.ws, kept_row(L), dy, ldy, dW, a);
    if (st != KFAC_OK) return st;
    if (kept_scratch(L, experts, n, fan, type) > c.ws_bytes) return KFAC_ERR_WORKSPACE;
    return run_kept(ctx, EXPERT_GRAD_WEIGHT, a, L, type, q, ldq, scales, lds);
}

kfac_status kfac_stats_expert_kept(kfac_ctx *ctx, const kfac_layer *L, int32_t experts, int32_t n, int32_t fan, kfac_dtype in,
                                   const int32_t *order, const int32_t *offsets, const uint8_t *q, int64_t ldq, const uint8_t *scales,
                                   int64_t lds, const void *grad_out, int64_t ldg, float decay, float *A_ema, float *G_ema)
{
    if (!expert_ok(ctx, L, experts, n, fan, in, offsets) || (A_ema && !kept_ok(L, n, fan, q, ldq, scales, lds))) return KFAC_ERR_INVALID;
    const CtxView c = ctx_view(ctx);
    ExpertArgs a;
    const kfac_status st = stats_args(ctx, L, experts, n, fan, in, order, offsets, A_ema ? kept_inputs(L, n, fan, q, ldq, scales, lds) : Inputs{}, c.ws,
                                      kept_row(L), grad_out, ldg, decay, A_ema, G_ema, a);
    if (st != KFAC_OK) return st;
    if (n == 0) return KFAC_OK;   // no expert has rows
    if (A_ema && kept_scratch(L, experts, n, fan, in) > c.ws_bytes) return KFAC_ERR_WORKSPACE;
    if (G_ema) {   // as ever: its input was not kept
        ExpertArgs g = a;
        g.A = nullptr;
        const kfac_status done = run_stats(ctx, g, in);
        if (done != KFAC_OK || !A_ema) return done;
    }
    a.G = nullptr;
    return run_kept(ctx, EXPERT_STATS, a, L, in, q, ldq, scales, lds);
}

}  // extern "C"
