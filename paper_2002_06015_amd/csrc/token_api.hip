// C entry points of the token and expert layers: segments, embedding, dropout, products grouped by expert and their factors.
// Argument checks, workspace, launches; no tables and no internal streams: everything goes to the context's stream.
#include <math.h>

#include <algorithm>

#include "token_internal.h"

using namespace kfac;

namespace {

constexpr int kMaxPositions = 1 << 30, kMaxDim = 1 << 20, kMaxExperts = 1 << 16;

bool type_ok(kfac_dtype t) { return t == KFAC_F32 || t == KFAC_BF16; }
size_t esize(kfac_dtype t) { return t == KFAC_BF16 ? 2 : 4; }

// Bytes that a call touches: one piece of `row` bytes every `ld` bytes from p to p + size; ld = 0: one piece.  Empty: touches nothing.
struct Range {
    const char *p;
    size_t size, row, ld;
    Range(const void *p_ = nullptr, size_t size_ = 0, size_t row_ = 0, size_t ld_ = 0) : p((const char *)p_), size(size_), row(ld_ ? row_ : size_), ld(ld_) {}
};
Range matrix(const void *p, long long rows, long long cols, long long ld, size_t es)
{
    if (!p || rows <= 0) return Range();
    return Range(p, (size_t)((rows - 1) * ld + cols) * es, (size_t)cols * es, rows > 1 && ld > cols ? (size_t)ld * es : 0);
}
// Columns beside each other in one wider tensor are apart though their ranges meet: with the same distance of rows (or one piece on
// one side) the two sets of pieces are compared inside one distance.
bool overlap(const Range &a, const Range &b)
{
    if (!a.size || !b.size || a.p >= b.p + b.size || b.p >= a.p + a.size) return false;
    if (a.ld != b.ld && a.ld && b.ld) return true;
    const size_t ld = a.ld ? a.ld : b.ld;
    if (!ld) return true;
    const size_t at = a.p <= b.p ? (size_t)(b.p - a.p) % ld : (ld - (size_t)(a.p - b.p) % ld) % ld;   // of b's pieces behind a's
    return at < a.row || at + b.row > ld;
}
// rows that lie ld elements apart: offsets, in bytes too, stay far inside 64 bits
bool spread_ok(long long rows, long long ld)
{
    constexpr long long most = 1LL << 40;
    return ld <= most && (rows <= 1 || ld <= most / rows);
}
bool aligned(const void *p, size_t es) { return (uintptr_t)p % es == 0; }

// One launch between the profiler's events
template <typename F>
bool timed(kfac_ctx *ctx, int kernel, int variant, double flops, double bytes, F launch)
{
    return profile_begin(ctx, kernel, variant, flops, bytes) && launch() == hipSuccess && profile_end(ctx);
}

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
    return timed(ctx, KFAC_K_EXPERT, (int)op, flops, bytes, [&] { return launch_expert(op, a, type == KFAC_BF16, c.fp32_planes, c.stream); });
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
    if (!expert_ok(ctx, L, experts, n, fan, type, offsets) || !aligned(order, 4) || !dW || !aligned(dW, 4)) return KFAC_ERR_INVALID;
    if (ldx < L->c_in || ldy < L->c_out || ldx > kMaxPositions || ldy > kMaxPositions) return KFAC_ERR_INVALID;
    const size_t es = esize(type);
    if (n > 0 && (!x || !dy || !aligned(x, es) || !aligned(dy, es))) return KFAC_ERR_INVALID;
    const Range out = matrix(dW, (long long)experts * L->c_out, L->c_in + L->bias, L->c_in + L->bias, 4);
    if (overlap(out, matrix(x, n / fan, L->c_in, ldx, es)) || overlap(out, matrix(dy, n, L->c_out, ldy, es))) return KFAC_ERR_INVALID;
    ExpertArgs a = expert_args(L, experts, n, fan, order, offsets);
    a.x = x; a.ldx = ldx; a.dy = dy; a.ldy = ldy; a.dW = dW;
    return run_expert(ctx, EXPERT_GRAD_WEIGHT, a, type, 2.0 * n * L->c_in * L->c_out,
                      es * (double)n * (L->c_in / (double)fan + L->c_out) + 4.0 * experts * L->c_out * (L->c_in + L->bias)) ? KFAC_OK : KFAC_ERR_DEVICE;
}

kfac_status kfac_stats_expert(kfac_ctx *ctx, const kfac_layer *L, int32_t experts, int32_t n, int32_t fan, kfac_dtype in, const int32_t *order,
                              const int32_t *offsets, const void *x, int64_t ldx, const void *grad_out, int64_t ldg, float decay, float *A_ema,
                              float *G_ema)
{
    if (!expert_ok(ctx, L, experts, n, fan, in, offsets) || !aligned(order, 4)) return KFAC_ERR_INVALID;
    if (!(decay >= 0.f && decay < 1.f) || (!A_ema && !G_ema) || !aligned(A_ema, 4) || !aligned(G_ema, 4)) return KFAC_ERR_INVALID;
    const size_t es = esize(in);
    if (A_ema && (ldx < L->c_in || ldx > kMaxPositions || (n > 0 && (!x || !aligned(x, es))))) return KFAC_ERR_INVALID;
    if (G_ema && (ldg < L->c_out || ldg > kMaxPositions || (n > 0 && (!grad_out || !aligned(grad_out, es))))) return KFAC_ERR_INVALID;
    const long long dA = L->c_in + L->bias, dG = L->c_out;
    const Range rx = A_ema ? matrix(x, n / fan, L->c_in, ldx, es) : Range{}, rg = G_ema ? matrix(grad_out, n, L->c_out, ldg, es) : Range{},
                A = matrix(A_ema, experts * dA, dA, dA, 4), G = matrix(G_ema, experts * dG, dG, dG, 4);
    if (overlap(A, G) || overlap(A, rx) || overlap(A, rg) || overlap(G, rx) || overlap(G, rg)) return KFAC_ERR_INVALID;
    if (n == 0) return KFAC_OK;   // no expert has rows
    ExpertArgs a = expert_args(L, experts, n, fan, order, offsets);
    a.x = x; a.ldx = ldx; a.dy = grad_out; a.ldy = ldg;
    a.A = A_ema; a.G = G_ema; a.decay = decay;
    const double fa = A_ema ? (double)dA * dA : 0.0, fg = G_ema ? (double)dG * dG : 0.0;
    return run_expert(ctx, EXPERT_STATS, a, in, n * (fa + fg), (double)rx.size + rg.size + 4.0 * experts * (fa + fg)) ? KFAC_OK
                                                                                                                               : KFAC_ERR_DEVICE;
}

}  // extern "C"
