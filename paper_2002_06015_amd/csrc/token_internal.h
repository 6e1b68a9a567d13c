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
};
enum ExpertOp { EXPERT_FORWARD, EXPERT_GRAD_INPUT, EXPERT_GRAD_WEIGHT, EXPERT_STATS };
// planes: how fp32 operands are multiplied (bf16 != 0: not used)
hipError_t launch_expert(ExpertOp op, const ExpertArgs &a, int bf16, bool planes, hipStream_t s);

}  // namespace kfac
