// What the entry points of the token and expert layers (token_api.hip) share with their kernel files.
// Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/kfac.h"
#include "kfac_internal.h"

namespace kfac {

// ---- the context, as seen from outside kfac_api.hip ---------------------------------------------------
struct CtxView {
    hipStream_t stream;
    char *ws;
    size_t ws_bytes;
    bool fp32_planes;   // fp32 products: planes, or the fp32 matrix instruction
};
CtxView ctx_view(const kfac_ctx *ctx);
// around one entry of the profile: records its times while profiling is on (nothing otherwise); false: a HIP call failed
bool profile_begin(kfac_ctx *ctx, int kernel, int variant, double flops, double bytes);
bool profile_end(kfac_ctx *ctx);

// ---- segments: a stable sort of positions by a small key ----------------------------------------------
// One workgroup sorts up to kSegSmall positions in LDS; more go through passes of a counting sort over tiles of kSegTile positions,
// kSegBits bits of the key a pass at most.
constexpr int kSegSmall = 8192, kSegTile = 2048, kSegBits = 9;
struct SegmentScratch {
    int *keys[2], *pos[2];   // [n] each: sorted keys and positions; pos[1] is not needed for n <= kSegSmall
    int *counts, *totals;    // [tiles << bits], [1 << bits] at least
    int passes, bits;        // of the counting sort
};
// Carves the scratch from `base` (nullptr: only counts); returns the bytes, which never fall as n or num grows.
size_t segment_scratch(char *base, int n, int num, SegmentScratch *out);
// Work that shares the sort's launches: data[0 .. count) <- 0 (unless nullptr), decayed[0 .. n_decayed) *= decay (without reading
// it for 0).  The sort keeps few CUs busy; the rest writes meanwhile.
struct Fill {
    float *data;
    long long count;
    float *decayed;
    int n_decayed;
    float decay;
};
// order: dev [n]; keys: the sorted keys end up there; offsets: dev [num + 1] or nullptr; fill: or nullptr
hipError_t launch_segments(const void *ids, int id_bits, int n, int num, const SegmentScratch &w, int *order, const int **keys,
                           int *offsets, const Fill *fill, hipStream_t s);
hipError_t launch_fill(const Fill &fill, hipStream_t s);

// ---- embedding -----------------------------------------------------------------------------------------
hipError_t launch_embedding(const void *ids, int id_bits, int n, int vocab, int dim, int table_bf16, const void *table, long long ldt,
                            float scale, int out_bf16, void *out, long long ldo, hipStream_t s);
struct EmbeddingGrad {
    const int *keys, *pos;   // sorted tokens and where they stand; keys >= vocab: no token
    int n, vocab, dim;
    const void *g;
    long long ld;
    int bf16, accumulate;
    float scale, share;      // share: (1 - decay) / n
    float *dW, *A;           // rows of zeros unless accumulate; decayed already, or nullptr
    float *partial;          // [2 * chunks][dim] at least
    int chunk;               // sorted positions that one wave adds up
};
int embedding_chunk(int n);
int embedding_most_chunks(int n);   // runs of any number of positions up to n
hipError_t launch_embedding_sum(const EmbeddingGrad &a, hipStream_t s);
hipError_t launch_embedding_join(const EmbeddingGrad &a, hipStream_t s);

// ---- dropout -------------------------------------------------------------------------------------------
struct DropoutArgs {
    long long rows, cols;
    const void *x, *r;       // r may be nullptr
    void *y;
    long long ldx, ldr, ldy;
    unsigned threshold;      // kept: 16 bits >= threshold
    float factor;
    unsigned long long seed, offset;
};
hipError_t launch_dropout(const DropoutArgs &a, int bf16, hipStream_t s);

// ---- products grouped by expert ------------------------------------------------------------------------
struct ExpertArgs {
    const int *order, *offsets;   // order may be nullptr: choice s is position s
    int n, experts, fan;
    int ci, co, bias;
    const void *x, *dy, *W;
    long long ldx, ldy, ldw;
    void *out;                    // y, dx
    long long ldo;
    float *dW;                    // [experts, co, ci + bias]
    float *A, *G;                 // [experts, ci + bias, ci + bias], [experts, co, co]
    float decay;
    float *partial;               // sums of pieces (launch_expert_pieces), expert_pieces_bytes of them
    int piece, most, whole_pieces;   // set by it: rows that an expert has at most if they are not cut, places for pieces, whether an XCD has whole ones
};
enum ExpertOp { EXPERT_FORWARD, EXPERT_GRAD_INPUT, EXPERT_GRAD_WEIGHT, EXPERT_STATS };
// planes: how fp32 operands are multiplied (bf16 != 0: not used)
hipError_t launch_expert(ExpertOp op, const ExpertArgs &a, int bf16, bool planes, hipStream_t s);

// The contractions over rows (gradient of the weights, factor A) for up to kPieceExperts experts, long ones cut into pieces; x is sorted: row s
// belongs to the choice at place s.
constexpr int kPieceExperts = 64;
size_t expert_pieces_bytes(int experts, int n, int ci, int co);   // never less for more rows, experts or channels
hipError_t launch_expert_pieces(ExpertOp op, const ExpertArgs &a, int bf16, bool planes, hipStream_t s);

// ---- routing -------------------------------------------------------------------------------------------
constexpr int kMaxRouted = 1024, kMaxFan = 32;
struct RouteArgs {
    int n, experts, fan, groups, top_groups, group_best, sigmoid, renormalise;
    float scale;
    const void *logits;
    long long ld;
    const float *bias;            // may be nullptr
    int *choice;
    float *gate;
    const float *dgate;           // of the gradient
    void *dlogits;
    long long ldd;
};
hipError_t launch_route(const RouteArgs &a, int bf16, hipStream_t s);
hipError_t launch_route_grad(const RouteArgs &a, int bf16, hipStream_t s);

// ---- the join of the experts' results ------------------------------------------------------------------
struct CombineArgs {
    int tokens, fan, dim;
    const void *y, *r, *dout;     // r may be nullptr
    long long ldy, ldr, ldd;
    const float *gate;            // may be nullptr
    void *out, *dy;               // dy may be nullptr
    long long ldo, lddy;
    float *dgate;                 // may be nullptr
};
hipError_t launch_combine(const CombineArgs &a, int bf16, int out_bf16, hipStream_t s);
hipError_t launch_combine_grad(const CombineArgs &a, int bf16, int out_bf16, hipStream_t s);

// ---- activations in 8 bits -----------------------------------------------------------------------------
struct KeepArgs {
    long long rows;
    int cols;
    bool gather;                  // of launch_restore: row s is that of the choice order[s] (or s), choice / fan
    const int *order;
    int fan;
    const void *x;                // of kfac_keep
    void *back;                   // of kfac_restore
    long long ldx;
    unsigned char *q, *scales;
    long long ldq, lds;
};
hipError_t launch_keep(const KeepArgs &a, int bf16, hipStream_t s);
hipError_t launch_restore(const KeepArgs &a, int bf16, hipStream_t s);

// ---- root-mean-square norm -----------------------------------------------------------------------------
constexpr int kMaxNorm = 16384;
struct NormArgs {
    int n, dim;
    const void *x, *r;            // r may be nullptr
    void *h, *y;                  // either may be nullptr
    const float *gamma;
    float eps;
    long long ldx, ldr, ldh, ldy;
    unsigned char *q, *scales;    // may be nullptr
    long long ldq, lds;
};
struct NormGradArgs {
    int n, dim;
    const void *dy, *h, *r;       // r: the stream's own gradient, may be nullptr
    void *dh;                     // may be nullptr
    long long lddy, ldh, ldr, lddh;
    const float *gamma;
    float eps;
    float *dgamma, *F;            // either may be nullptr
    float decay;
    float *partial;               // [parts][2][dim], not read or written if both are nullptr
};
hipError_t launch_norm(const NormArgs &a, int bf16, int stream_bf16, hipStream_t s);
int norm_parts(int n, int dim);   // never fewer for more rows or columns
hipError_t launch_norm_grad(const NormGradArgs &a, int bf16, int stream_bf16, hipStream_t s);
hipError_t launch_norm_join(const NormGradArgs &a, hipStream_t s);

}  // namespace kfac
