// Products grouped by expert: the rows of x that an expert received, as a segment of `order`, times its weights, and the
// gradients and Kronecker factors of the same rows.  With c = order[s] for the choices s of expert e's segment:
//   forward       y[c, :]  = x[c / fan, :] W_e^T (+ b_e)
//   grad_input    dx[c, :] = dy[c, :] W_e
//   grad_weight   dW_e     = sum_s dy[c, :]^T x[c / fan, :]                     (bias column: sum_s dy[c, :])
//   statistics    A_e = 1/n_e sum_s x x^T (with a constant-one row for the bias), G_e = 1/n_e sum_s dy dy^T
// The segments' lengths are known to the device only: a launch has as many workgroups as there can be tiles, and every
// workgroup finds its tile from the offsets (a wave adds up the experts' tile counts).  Rows are gathered and scattered
// through `order` where they are loaded and stored.
//
// All four are C(i, j) = sum_k a(i, k) b(j, k) with an operand stored along k (rows of x, dy or W) or across k (the
// contraction runs over rows of the tensor).  Tiles across k are kept in LDS as they lie in memory and reach the matrix
// instruction through the transposing LDS read (ds_read_b64_tr_b16: among 16 lanes, lane i receives element i % 4 of the four
// 8-byte groups addressed by lanes i / 4, i / 4 + 4, i / 4 + 8, i / 4 + 12).
// fp32 operands are the exact sum of three bf16 values; of the nine products the six above 2^-24 are formed (h h, h m, m h,
// m m, h l, l h), all accumulated in fp32.  Contexts that ask for the fp32 matrix instruction get it.
#include <algorithm>
#include <type_traits>

#include "gemm_tiles.h"
#include "lds_dma.h"
#include "token_internal.h"

namespace kfac {

namespace {

typedef unsigned short bf16_t;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) shortx4 *lds_shortx4_ptr;
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx4_u __attribute__((ext_vector_type(4), aligned(2)));                 // 16 bytes at an element's alignment
typedef float floatx4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short u16x4_u __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ bf16_t to_bf16(float v) { return __builtin_bit_cast(bf16_t, (__bf16)v); }

__device__ __forceinline__ floatx4 mfma(const bf16x8 &j, const bf16x8 &i, const floatx4 &c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(j, i, c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 mfma(float j, float i, const floatx4 &c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(j, i, c, 0, 0, 0); }

// ---- segments ------------------------------------------------------------------------------------------
__device__ __forceinline__ int segment_begin(const ExpertArgs &a, int e) { return min(max(a.offsets[e], 0), a.n); }
// e == experts: the choices that no expert takes
__device__ __forceinline__ void segment(const ExpertArgs &a, int e, int &begin, int &len)
{
    begin = segment_begin(a, e);
    len = max(e < a.experts ? segment_begin(a, e + 1) : a.n, begin) - begin;
}
// the choice at place s of the sorted list, -1 if there is none
__device__ __forceinline__ int choice_at(const ExpertArgs &a, int s)
{
    const int c = a.order ? a.order[s] : s;
    return c >= 0 && c < a.n ? c : -1;
}

// Tiles in bands of 4 rows, column by column: the 32 that an XCD works on at one time are 4 x 8 and touch 12 panels of operands.
__device__ __forceinline__ void banded(int local, int rows, int tiles_j, int &ti, int &tj)
{
    const int band = local / (4 * tiles_j), high = min(4, rows - 4 * band);
    local -= band * 4 * tiles_j;
    tj = local / high;
    ti = 4 * band + local - tj * high;
}

// Tile `block` of those of all experts with BM rows and tiles_j columns of tiles each; false: there are fewer.  Every XCD works through
// one contiguous share.  All threads of a wave call it.
template <int BM>
__device__ __forceinline__ bool find_tile(const ExpertArgs &a, int block, int tiles_j, int &e, int &begin, int &len, int &ti, int &tj)
{
    const int lane = threadIdx.x & 63;
    int total = 0;
    for (int e0 = 0; e0 <= a.experts; e0 += 64) {
        int b = 0, l = 0;
        if (e0 + lane <= a.experts) segment(a, e0 + lane, b, l);
        int t = (l + BM - 1) / BM;
        for (int o = 32; o > 0; o >>= 1) t += __shfl_xor(t, o);
        total += t;
    }
    total *= tiles_j;
    if (block >= total) return false;
    const int id = xcd_remap(block, total);
    int before = 0;
    for (int e0 = 0; e0 <= a.experts; e0 += 64) {
        int b = 0, l = 0;
        if (e0 + lane <= a.experts) segment(a, e0 + lane, b, l);
        const int t = (l + BM - 1) / BM * tiles_j;
        int incl = t;
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(incl, o);
            if (lane >= o) incl += up;
        }
        const unsigned long long has = __ballot(id < before + incl);
        if (has) {
            const int who = __ffsll(has) - 1;
            e = __builtin_amdgcn_readfirstlane(e0 + who);
            begin = __builtin_amdgcn_readlane(b, who);
            len = __builtin_amdgcn_readlane(l, who);
            banded(id - before - (__builtin_amdgcn_readlane(incl, who) - __builtin_amdgcn_readlane(t, who)), (len + BM - 1) / BM, tiles_j, ti, tj);
            return true;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
    }
    return false;
}

// ---- tiles in LDS --------------------------------------------------------------------------------------
// 16-byte chunks of 8 elements.  Along k: line = row of the tile, BK / 8 chunks; across k: line = k, ROWS / 8 chunks of 8 rows.
// Chunks are permuted inside a line so that the lanes of a read meet different banks.
template <bool ACROSS, int BK, int ROWS>
__device__ __forceinline__ int chunk_at(int line, int pos)
{
    if constexpr (ACROSS && ROWS == 64) return line * 8 + ((((pos >> 1) ^ (((line >> 1) & 1) | ((line >> 2) & 2))) << 1) | (pos & 1));
    else if constexpr (ACROSS) return line * (ROWS / 8) + ((((pos >> 1) ^ ((line & 3) | ((line >> 1) & 4))) << 1) | (pos & 1));
    else if constexpr (BK == 64) return line * 8 + (pos ^ (line & 7));
    else return line * 4 + (pos ^ ((line >> 1) & 3));
}

// The 16 rows from `row0` (a multiple of 16) of a tile, k = 32 u + 8 (lane / 16) .. + 7: lane -> row lane % 16.
template <bool ACROSS, int BK, int ROWS>
__device__ __forceinline__ bf16x8 fragment(const bf16_t *tile, int row0, int u, int lane)
{
    if constexpr (ACROSS) {
        const int m = 32 * u + 8 * (lane >> 4) + ((lane & 15) >> 2);
        const bf16_t *p = tile + 8 * chunk_at<true, BK, ROWS>(m, row0 / 8) + 4 * (lane & 3);   // (the pair of chunks stays together)
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_ptr)p);
        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_ptr)(p + 4 * ROWS));   // k + 4: same permutation
        return __builtin_bit_cast(bf16x8, shortx8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    } else {
        return *(const bf16x8 *)(tile + 8 * chunk_at<false, BK, ROWS>(row0 + (lane & 15), 4 * u + (lane >> 4)));
    }
}

// fp32 tiles of the fp32 matrix instruction: 32 k.  Where element (line, at) of a tile is; eight (along k: four) adjacent ones stay
// together, and the lanes of a read meet different banks.
template <bool ACROSS, int ROWS>
__device__ __forceinline__ int float_at(int line, int at)
{
    if constexpr (ACROSS) return line * ROWS + (at ^ (line & 12) << 2);
    else return line * 32 + (at ^ (line & 7) << 2);
}

// The 16 rows from `row0` of such a tile, k = 16 u + 4 (lane / 16) .. + 3: lane -> row lane % 16.
template <bool ACROSS, int ROWS>
__device__ __forceinline__ floatx4 fragment(const float *tile, int row0, int u, int lane)
{
    const int k = 16 * u + 4 * (lane >> 4), row = row0 + (lane & 15);
    if constexpr (ACROSS) {
        const float *p = tile + float_at<true, ROWS>(k, row);   // (the four lines are permuted alike)
        return floatx4{p[0], p[ROWS], p[2 * ROWS], p[3 * ROWS]};
    } else {
        return *(const floatx4 *)(tile + float_at<false, ROWS>(row, k));
    }
}

// ---- general kernel: any size, stride and alignment -----------------------------------------------------
// Tiles of 128 x 128 (four waves of 64 x 64) or 64 x 64 (of 32 x 32, several groups of waves that share the contraction); operands go
// through registers, and are converted there if they are fp32, while the next step's loads are in flight.  fp32: 177 - 195 TFLOP/s on 4096 rows
// 4096 -> 4096 (the library's product has 151), bound by the vector instructions that split the operands (6 of them for each matrix
// instruction in small tiles) and the matrix unit's power; bf16 with odd sizes 16384 rows 1025 -> 2049: 240 - 450 TFLOP/s.
// The fp32 instruction: 118 TFLOP/s of its 157 there (1160 us instead of 700 - 750), and 42, 48 and 45 us for the products of 2051 rows
// 515 -> 1000 of 8 even experts (34, 37 and 33 through planes): for its range, not for its speed.
template <typename T>
struct Chunk {
    uintx4 v[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p, int c)   // the first c elements, zeros behind them
    {
        if (c >= 8) {
            if constexpr (sizeof(T) == 2) {
                v[0] = *(const uintx4_u *)p;
            } else {
                v[0] = __builtin_bit_cast(uintx4, (floatx4)*(const floatx4_u *)p);
                v[1] = __builtin_bit_cast(uintx4, (floatx4)*(const floatx4_u *)(p + 4));
            }
            return;
        }
#pragma unroll
        for (int q = 0; q < (int)sizeof(T) / 2; ++q) v[q] = uintx4{0, 0, 0, 0};
        if (c <= 0) return;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < c) {
                if constexpr (sizeof(T) == 2) v[0][j >> 1] |= (unsigned)p[j] << (16 * (j & 1));
                else v[j >> 2][j & 3] = __float_as_uint(p[j]);
            }
    }
    // into the planes of a tile
    __device__ __forceinline__ void store(bf16_t *tile, int plane, int at) const
    {
        if constexpr (sizeof(T) == 2) {
            *(uintx4 *)(tile + 8 * at) = v[0];
        } else {
            uintx4 h, m, l;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                unsigned x, y, z;
                split_pair(__uint_as_float(v[q >> 1][2 * (q & 1)]), __uint_as_float(v[q >> 1][2 * (q & 1) + 1]), x, y, z);
                h[q] = x; m[q] = y; l[q] = z;
            }
            *(uintx4 *)(tile + 8 * at) = h;
            *(uintx4 *)(tile + plane + 8 * at) = m;
            *(uintx4 *)(tile + 2 * plane + 8 * at) = l;
        }
    }
    // into a tile of the fp32 instruction, four elements at each place
    __device__ __forceinline__ void store(float *at0, float *at1) const
    {
        static_assert(sizeof(T) == 4, "fp32 operands");
        *(uintx4 *)at0 = v[0];
        *(uintx4 *)at1 = v[1];
    }
};

// One operand of a tile.  Along k: rows [0, rows) from `line`; across k: columns col0 .. of `cols`, k < K.
// GATHER: 0: line r is base + r ld;  1: base + choice_at(begin + r) ld;  2: base + choice_at(begin + r) / fan * ld
// (fan: 1 where the rows are those of the choices)
template <typename T, bool ACROSS, int GATHER, int BK, int EDGE>
struct Staged {
    static constexpr int CH = BK * EDGE / 2048, PER = ACROSS ? EDGE / 8 : BK / 8;
    const T *base;
    long long ld;
    int begin, K, cols, col0;
    unsigned fan;
    const T *line_ptr[CH];   // along k
    int choice[CH];          // across k, gathered: the choices of the next step
    Chunk<T> reg[CH];

    __device__ __forceinline__ const T *line(int r, int c) const
    {
        if constexpr (GATHER == 0) return base + (long long)r * ld;
        else if constexpr (GATHER == 1) return base + (long long)c * ld;
        else return base + (long long)((unsigned)c / fan) * ld;
    }
    __device__ __forceinline__ void next_choices(const ExpertArgs &a, int k0, int tid)
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int k = k0 + (tid + 256 * i) / PER;
            choice[i] = k < K ? choice_at(a, begin + k) : -1;
        }
    }
    // rows: of the tile's first row on (along k); cols and K as above; k0: the first step
    __device__ __forceinline__ void init(const ExpertArgs &a, const T *base_, long long ld_, int fan_, int begin_, int row0, int rows, int K_, int k0, int tid)
    {
        base = base_; ld = ld_; fan = (unsigned)fan_; begin = begin_; K = K_; cols = rows; col0 = row0;
        if constexpr (!ACROSS) {
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int r = row0 + (tid + 256 * i) / PER;
                int c = 0;
                if constexpr (GATHER != 0) c = r < rows ? choice_at(a, begin + r) : -1;
                line_ptr[i] = r < rows && c >= 0 ? line(r, c) : nullptr;
            }
        } else if constexpr (GATHER != 0) {
            next_choices(a, k0, tid);
        }
    }
    __device__ __forceinline__ void load(const ExpertArgs &a, int k0, int apart, int tid)   // the next one: apart further
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int q = tid + 256 * i, pos = 8 * (q % PER);
            if constexpr (!ACROSS) {
                reg[i].load(line_ptr[i] + k0 + pos, line_ptr[i] ? K - k0 - pos : 0);
            } else {
                const int k = k0 + q / PER;
                bool there = k < K;
                int c = 0;
                if constexpr (GATHER != 0) { c = choice[i]; there = c >= 0; }
                reg[i].load(there ? line(k, c) + col0 + pos : base, there ? cols - col0 - pos : 0);
            }
        }
        if constexpr (ACROSS && GATHER != 0) next_choices(a, k0 + apart, tid);
    }
    __device__ __forceinline__ void store(bf16_t *tile, int tid) const
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int q = tid + 256 * i;
            reg[i].store(tile, EDGE * BK, chunk_at<ACROSS, BK, EDGE>(q / PER, q % PER));
        }
    }
    __device__ __forceinline__ void store(float *tile, int tid) const
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int q = tid + 256 * i, line = q / PER, at = 8 * (q % PER);
            reg[i].store(tile + float_at<ACROSS, EDGE>(line, at), tile + float_at<ACROSS, EDGE>(line, at + 4));
        }
    }
};

template <typename T>
__device__ __forceinline__ void store4(T *p, int c, const floatx4 &v)   // the first c of four adjacent elements
{
    if constexpr (sizeof(T) == 2) {
        if (c >= 4) {
            *(u16x4_u *)p = u16x4_u{to_bf16(v[0]), to_bf16(v[1]), to_bf16(v[2]), to_bf16(v[3])};
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r < c) p[r] = to_bf16(v[r]);
        }
    } else {
        if (c >= 4) {
            *(floatx4_u *)p = v;
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r < c) p[r] = v[r];
        }
    }
}

__device__ __forceinline__ float blend(float decay, float alpha, float old, float sum)
{
    return decay == 0.f ? alpha * sum : fmaf(alpha, sum, decay * old);
}

// What a workgroup works on: C(i, j) for rows from ti BM and columns from tj BN, i < I, j < J, contraction over K.
struct Tile {
    int e, begin, len, ti, tj, I, J, K;
    bool g;   // statistics: G_e
};

// Tiles of the lower triangle of a symmetric matrix.
template <int EDGE>
__host__ __device__ __forceinline__ int triangle_tiles(int dim)
{
    const int t = (dim + EDGE - 1) / EDGE;
    return t * (t + 1) / 2;
}

// Contractions over the rows of an expert take as long as it has rows: every XCD gets an eighth of every expert's tiles.
// slots: workgroups an expert, a multiple of 8, at least `tiles`.
__device__ __forceinline__ bool expert_share(int slots, int tiles, int &e, int &local)
{
    const int x = blockIdx.x & 7, q = blockIdx.x >> 3, per = slots >> 3;
    e = q / per;
    local = x * per + q - e * per;
    return local < tiles;
}

// Tile `local` of an expert's, for the contractions over rows.
template <int OP, int BM, int BN>
__device__ __forceinline__ void row_tile(const ExpertArgs &a, int tiles_j, int local, Tile &t)
{
    t.g = false;
    if constexpr (OP == EXPERT_GRAD_WEIGHT) {
        banded(local, (a.co + BM - 1) / BM, tiles_j, t.ti, t.tj);
        t.I = a.co;
        t.J = a.ci;
    } else {
        static_assert(BM == BN, "the triangle has square tiles");
        tri_decode(local, t.ti, t.tj);
        t.I = t.J = a.ci;
    }
}

// Contractions over rows in pieces (up to 64 experts; of the statistics factor A alone; x sorted: row s is that of the choice at place s): the rows
// of an expert that has more than a.piece of them are cut into equal parts, and the parts of all experts are taken up in the order of their
// lengths, so that the last ones to run are short ones (16 uneven experts: weights 137 -> 133 us, factors 186 -> 176).  Lane e of every
// wave knows expert e's.
struct Pieces {
    int begin, len, count, rows;   // of the expert; its pieces and their rows (the last has what is left)
    int first, slot;               // places of its first piece: in the order of lengths; among the pieces of experts with several
    int split;                     // experts before it that have several
};
template <int OP>
__device__ __forceinline__ Pieces pieces_of(const ExpertArgs &a)
{
    const int lane = threadIdx.x & 63;
    Pieces p{};
    if (lane < a.experts) {
        segment(a, lane, p.begin, p.len);
        const int want = (p.len + a.piece - 1) / a.piece;
        p.rows = want > 1 ? ((p.len + want - 1) / want + 63) / 64 * 64 : p.len;
        p.count = want > 1 ? (p.len + p.rows - 1) / p.rows : OP == EXPERT_GRAD_WEIGHT || p.len > 0 ? 1 : 0;   // (weights without rows become zero)
    }
    for (int e = 0; e < a.experts; ++e) {
        const int rows = __builtin_amdgcn_readlane(p.rows, e), count = __builtin_amdgcn_readlane(p.count, e);
        p.first += rows > p.rows || (rows == p.rows && e < lane) ? count : 0;
        if (e < lane && count > 1) { p.slot += count; ++p.split; }
    }
    return p;
}
// slot: where the tile's sums go, -1: straight into the result
template <int OP, int BM, int BN>
__device__ __forceinline__ bool find_piece(const ExpertArgs &a, int tiles_j, int tiles, Tile &t, int &slot)
{
    const Pieces p = pieces_of<OP>(a);
    // of every piece an XCD has an eighth of the tiles, or it has whole pieces, in turn forth and back
    const int x = blockIdx.x & 7, i = blockIdx.x >> 3, per = a.whole_pieces ? tiles : (tiles + 7) / 8;
    const int round = i / per, at = !a.whole_pieces ? round : 8 * round + (round & 1 ? 7 - x : x), local = (a.whole_pieces ? 0 : x * per) + i - round * per;
    const unsigned long long has = __ballot(at >= p.first && at < p.first + p.count);
    if (!has || local >= tiles) return false;
    const int e = __ffsll(has) - 1;
    const int rows = __builtin_amdgcn_readlane(p.rows, e), count = __builtin_amdgcn_readlane(p.count, e), q = at - __builtin_amdgcn_readlane(p.first, e);
    t.e = e;
    t.len = __builtin_amdgcn_readlane(p.len, e);
    t.begin = __builtin_amdgcn_readlane(p.begin, e) + q * rows;
    t.K = min(rows, t.len - q * rows);
    const int place = __builtin_amdgcn_readlane(p.slot, e) + q;
    if (count > 1 && place >= a.most) return false;   // (offsets that no sort makes: segments that overlap)
    slot = count > 1 ? place * tiles + local : -1;
    row_tile<OP, BM, BN>(a, tiles_j, local, t);
    return true;
}
// What a tile's sums take in the workspace: the sums in the order of the kernel's registers, then those of its rows.
template <int BM, int BN>
__host__ __device__ constexpr long long slot_floats() { return (long long)BM * BN + BM; }

template <int OP, int BM, int BN>
__device__ __forceinline__ bool find_work(const ExpertArgs &a, int tiles_j, int total, Tile &t)
{
    t.g = false;
    if constexpr (OP == EXPERT_FORWARD || OP == EXPERT_GRAD_INPUT) {
        if (!find_tile<BM>(a, blockIdx.x, tiles_j, t.e, t.begin, t.len, t.ti, t.tj)) return false;
        t.I = t.len;
        t.J = OP == EXPERT_FORWARD ? a.co : a.ci;
        t.K = t.e == a.experts ? 0 : OP == EXPERT_FORWARD ? a.ci : a.co;   // rows of choices that no expert takes are zero
        return true;
    } else if constexpr (OP == EXPERT_GRAD_WEIGHT) {
        const int tiles_i = (a.co + BM - 1) / BM;
        int local;
        if (!expert_share(total / a.experts, tiles_i * tiles_j, t.e, local)) return false;
        banded(local, tiles_i, tiles_j, t.ti, t.tj);
        segment(a, t.e, t.begin, t.len);
        t.I = a.co; t.J = a.ci; t.K = t.len;
        return true;
    } else {
        const int na = a.A ? triangle_tiles<BM>(a.ci) : 0, per = na + (a.G ? triangle_tiles<BM>(a.co) : 0);
        int local;
        if (!expert_share(total / a.experts, per, t.e, local)) return false;
        t.g = local >= na;
        if (t.g) local -= na;
        static_assert(BM == BN, "the triangle has square tiles");
        tri_decode(local, t.ti, t.tj);
        segment(a, t.e, t.begin, t.len);
        t.I = t.J = t.g ? a.co : a.ci;
        t.K = t.len;
        return t.len > 0;   // an expert without rows keeps its factors
    }
}

// Whether a wave adds up its rows over k besides: the bias column of dW, the border of A.
template <int OP>
__device__ __forceinline__ bool wants_sums(const ExpertArgs &a, const Tile &t, int wj)
{
    return (OP == EXPERT_GRAD_WEIGHT || OP == EXPERT_STATS) && a.bias && !t.g && t.tj == 0 && wj == 0;
}

// Row and column ci of A_e, and its corner: the bias.
__device__ __forceinline__ void store_border(const ExpertArgs &a, const Tile &t, int row, float sum)
{
    const int d = a.ci + a.bias;
    float *M = a.A + (long long)t.e * d * d, *lo = M + (long long)a.ci * d + row;
    const float v = blend(a.decay, (1.f - a.decay) / (float)t.len, a.decay == 0.f ? 0.f : *lo, sum);
    *lo = v;
    M[(long long)row * d + a.ci] = v;
    if (row == 0) {
        float *corner = M + (long long)a.ci * d + a.ci;
        *corner = blend(a.decay, 1.f - a.decay, a.decay == 0.f ? 0.f : *corner, 1.f);
    }
}

__device__ __forceinline__ float value(bf16_t v) { return __uint_as_float((unsigned)v << 16); }
__device__ __forceinline__ float value(float v) { return v; }

// Stores a BM x BN tile whose sums are spread over the workgroup's registers.  They go out through LDS, PART rows at a time, so
// that a wave stores whole pieces of rows: straight from the registers a store would touch 16 to 32 bytes of each of 16 or 32 rows
// (65536 rows 64 -> 2048 in bf16: 213 us instead of 92).  put(p0): brings rows p0 .. p0 + PART - 1 into `part`, rows LD apart, with
// what put_quad gives for four adjacent sums.
template <typename T, int OP, int BM, int BN, int PART, int THREADS, typename Put>
__device__ __forceinline__ void store_rows(const ExpertArgs &a, const Tile &t, void *memory, int tid, Put put)
{
    const int i0 = t.ti * BM, j0 = t.tj * BN;
    if constexpr (OP == EXPERT_FORWARD || OP == EXPERT_GRAD_INPUT) {
        constexpr int E = 16 / sizeof(T), LD = BN + E, PER_ROW = BN / E, ROWS = THREADS / PER_ROW;   // 16-byte pieces
        T *const part = (T *)memory;
        const int col = E * (tid % PER_ROW), left = t.J - j0 - col;
        for (int p0 = 0; p0 < BM && i0 + p0 < t.I; p0 += PART) {
            __syncthreads();
            put(p0, [&](int row, int c, const floatx4 &v) {
                floatx4 w = v;
                if (OP == EXPERT_FORWARD && a.bias && t.e < a.experts) {
                    const T *bias = (const T *)a.W + ((long long)t.e * a.co + j0 + c) * a.ldw + a.ci;
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (j0 + c + r < t.J) w[r] += value(bias[(long long)r * a.ldw]);
                }
                store4<T>(part + (row - p0) * LD + c, 4, w);
            });
            __syncthreads();
#pragma unroll 4
            for (int r = tid / PER_ROW; r < PART; r += ROWS) {
                if (i0 + p0 + r >= t.I) break;
                const int c = choice_at(a, t.begin + i0 + p0 + r);
                const uintx4 v = *(const uintx4 *)(part + r * LD + col);
                T *out = (T *)a.out + (long long)c * a.ldo + j0 + col;
                if (c >= 0 && left >= E) {
                    *(uintx4_u *)out = v;
                } else if (c >= 0) {
#pragma unroll
                    for (int q = 0; q < E; ++q)
                        if (q < left) out[q] = part[r * LD + col + q];
                }
            }
        }
    } else {
        constexpr int LD = BN + 4, PER_ROW = BN / 4, ROWS = THREADS / PER_ROW;
        constexpr bool w = OP == EXPERT_GRAD_WEIGHT;
        float *const part = (float *)memory;
        const int d = w ? a.ci + a.bias : t.g ? a.co : a.ci + a.bias;
        float *const M = w ? a.dW + (long long)t.e * a.co * d : (t.g ? a.G : a.A) + (long long)t.e * d * d;
        const float alpha = w ? 1.f : (1.f - a.decay) / (float)t.len;
        const int col = 4 * (tid % PER_ROW);
        for (int p0 = 0; p0 < BM && i0 + p0 < t.I; p0 += PART) {
            __syncthreads();
            put(p0, [&](int row, int c, const floatx4 &v) { *(floatx4 *)(part + (row - p0) * LD + c) = v; });
            __syncthreads();
            for (int r = tid / PER_ROW; r < PART && i0 + p0 + r < t.I; r += ROWS) {
                const int row = i0 + p0 + r, left = (w ? t.J : min(t.J, row + 1)) - j0 - col;   // (of factors the lower triangle)
                if (left <= 0) continue;
                float *out = M + (long long)row * d + j0 + col;
                floatx4 v = *(const floatx4 *)(part + r * LD + col);
                if constexpr (!w) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[q] = blend(a.decay, alpha, a.decay != 0.f && q < left ? out[q] : 0.f, v[q]);
                    *(floatx4 *)(part + r * LD + col) = v;
                }
                store4<float>(out, left, v);
            }
            if constexpr (!w) {   // the mirror image: lanes along the rows
                __syncthreads();
                for (int u = tid; u < BN * PART; u += THREADS) {
                    const int r = u % PART, c = u / PART, row = i0 + p0 + r;
                    if (row < t.I && row > j0 + c) M[(long long)(j0 + c) * d + row] = part[r * LD + c];
                }
            }
        }
    }
}

// The sum of a row over k: the bias column of dW, or the border of A_e.
template <int OP>
__device__ __forceinline__ void store_sum(const ExpertArgs &a, const Tile &t, int row, float sum)
{
    if (row >= t.I) return;
    if constexpr (OP == EXPERT_GRAD_WEIGHT) a.dW[((long long)t.e * a.co + row) * (a.ci + a.bias) + a.ci] = sum;
    else if constexpr (OP == EXPERT_STATS) store_border(a, t, row, sum);
}

// The product with ones adds up the second operand's rows over k, into every row of the result.  (Ones in one row and zeros in the
// others would let several blocks share a result, but a zero times an infinity or a NaN is a NaN in the sums of another block.)
__device__ __forceinline__ floatx4 add_up(const bf16x8 &i, const floatx4 &c)
{
    constexpr unsigned one = 0x3F803F80u;
    return mfma(__builtin_bit_cast(bf16x8, uintx4{one, one, one, one}), i, c);
}

// GROUPS of four waves share a tile: each takes every GROUPS-th step of the contraction, the sums are added up in the groups' order.
// FP32: with the fp32 matrix instruction, whose four k of step v are 16 u + 4 q + v of the lanes 16 q .. 16 q + 15.
template <typename T, bool FP32, int OP, int EDGE, int GROUPS, bool PIECES>
__global__ __launch_bounds__(256 * GROUPS, EDGE == 128 ? 2 : 4) void expert_general_kernel(const ExpertArgs a, int tiles_j, int total)
{
    typedef std::conditional_t<FP32, float, bf16_t> E;   // what is in LDS
    constexpr int BK = sizeof(T) == 2 ? 64 : 32, NP = sizeof(T) == 2 || FP32 ? 1 : 3;
    constexpr bool ACROSS_A = OP == EXPERT_GRAD_WEIGHT || OP == EXPERT_STATS;
    constexpr bool ACROSS_B = OP != EXPERT_FORWARD;
    constexpr int GATHER_X = PIECES ? 0 : 2;
    constexpr int GATHER_A = OP == EXPERT_FORWARD ? 2 : OP == EXPERT_STATS ? GATHER_X : 1;
    constexpr int GATHER_B = OP == EXPERT_GRAD_WEIGHT || OP == EXPERT_STATS ? GATHER_X : 0;
    constexpr int PLANE = EDGE * BK, NB = EDGE / 32;   // NB x NB blocks of 16 x 16 a wave
    __shared__ __attribute__((aligned(16))) E lds[GROUPS * 2 * NP * PLANE];
    const int tid = threadIdx.x & 255, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = GROUPS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0, first = group * BK;
    const int wi = wave >> 1, wj = wave & 1;
    E *const tile_a = lds + group * 2 * NP * PLANE, *const tile_b = tile_a + NP * PLANE;
    Tile t;
    int slot = -1;
    if constexpr (PIECES) {
        if (!find_piece<OP, EDGE, EDGE>(a, tiles_j, total, t, slot)) return;
    } else {
        if (!find_work<OP, EDGE, EDGE>(a, tiles_j, total, t)) return;
    }

    Staged<T, ACROSS_A, GATHER_A, BK, EDGE> sa;
    Staged<T, ACROSS_B, GATHER_B, BK, EDGE> sb;
    const T *We = (const T *)a.W + (long long)min(t.e, a.experts - 1) * a.co * a.ldw, *x = (const T *)a.x + (PIECES ? t.begin * a.ldx : 0), *dy = (const T *)a.dy;
    if constexpr (OP == EXPERT_FORWARD) sa.init(a, x, a.ldx, a.fan, t.begin, t.ti * EDGE, t.I, t.K, first, tid);
    else if constexpr (OP == EXPERT_STATS) sa.init(a, t.g ? dy : x, t.g ? a.ldy : a.ldx, t.g ? 1 : a.fan, t.begin, t.ti * EDGE, t.I, t.K, first, tid);
    else sa.init(a, dy, a.ldy, 1, t.begin, t.ti * EDGE, t.I, t.K, first, tid);
    if constexpr (OP == EXPERT_FORWARD || OP == EXPERT_GRAD_INPUT) sb.init(a, We, a.ldw, 1, 0, t.tj * EDGE, t.J, t.K, first, tid);
    else if constexpr (OP == EXPERT_STATS) sb.init(a, t.g ? dy : x, t.g ? a.ldy : a.ldx, t.g ? 1 : a.fan, t.begin, t.tj * EDGE, t.J, t.K, first, tid);
    else sb.init(a, x, a.ldx, a.fan, t.begin, t.tj * EDGE, t.J, t.K, first, tid);
    const bool sums = wants_sums<OP>(a, t, wj);

    floatx4 acc[NB][NB], row_sum[NB];   // row_sum[i][0] of lanes 0 .. 15: the rows of block i
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        row_sum[i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    auto load = [&](int k0) {
        if (k0 < t.K) {
            sa.load(a, k0, GROUPS * BK, tid);
            sb.load(a, k0, GROUPS * BK, tid);
        }
    };
    auto multiply = [&]() {
        if constexpr (FP32) {
#pragma unroll
            for (int u = 0; u < BK / 16; ++u) {
                floatx4 fa[NB], fb[NB];
#pragma unroll
                for (int q = 0; q < NB; ++q) {
                    fa[q] = fragment<ACROSS_A, EDGE>(tile_a, wi * (EDGE / 2) + 16 * q, u, lane);
                    fb[q] = fragment<ACROSS_B, EDGE>(tile_b, wj * (EDGE / 2) + 16 * q, u, lane);
                }
#pragma unroll
                for (int v = 0; v < 4; ++v) {
#pragma unroll
                    for (int i = 0; i < NB; ++i)
#pragma unroll
                        for (int j = 0; j < NB; ++j) acc[i][j] = mfma(fb[j][v], fa[i][v], acc[i][j]);
                    if (sums)
#pragma unroll
                        for (int i = 0; i < NB; ++i) row_sum[i] = mfma(1.f, fa[i][v], row_sum[i]);
                }
            }
        } else {
#pragma unroll
            for (int u = 0; u < BK / 32; ++u) {
                bf16x8 fa[NP][NB], fb[NP][NB];
#pragma unroll
                for (int p = 0; p < NP; ++p)
#pragma unroll
                    for (int q = 0; q < NB; ++q) {
                        fa[p][q] = fragment<ACROSS_A, BK, EDGE>(tile_a + p * PLANE, wi * (EDGE / 2) + 16 * q, u, lane);
                        fb[p][q] = fragment<ACROSS_B, BK, EDGE>(tile_b + p * PLANE, wj * (EDGE / 2) + 16 * q, u, lane);
                    }
                constexpr int pa[6] = {0, 2, 1, 0, 1, 0}, pb[6] = {2, 0, 1, 1, 0, 0};   // the small products first
#pragma unroll
                for (int q = NP == 1 ? 5 : 0; q < 6; ++q)
#pragma unroll
                    for (int i = 0; i < NB; ++i)
#pragma unroll
                        for (int j = 0; j < NB; ++j) acc[i][j] = mfma(fb[pb[q]][j], fa[pa[q]][i], acc[i][j]);
                if (sums)
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                        for (int i = 0; i < NB; ++i) row_sum[i] = add_up(fa[p][i], row_sum[i]);
            }
        }
    };
    load(first);
    for (int k0 = 0; k0 < t.K; k0 += GROUPS * BK) {
        if (k0 > 0) __syncthreads();   // every wave has read the step before
        if (k0 + first < t.K) {
            sa.store(tile_a, tid);
            sb.store(tile_b, tid);
        }
        __syncthreads();
        load(k0 + first + GROUPS * BK);
        if (k0 + first < t.K) multiply();
    }
    if constexpr (GROUPS > 1) {
        constexpr int LD = EDGE + 4;
        static_assert((EDGE * LD + EDGE) * 4 <= sizeof(lds), "a group's sums have to fit");
        float *const part = (float *)lds, *const part_rows = part + EDGE * LD;
        for (int g = 1; g < GROUPS; ++g) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int row = wi * (EDGE / 2) + 16 * i + (lane & 15);
                if (group == g && sums && lane < 16) part_rows[row] = row_sum[i][0];
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    if (group == g) *(floatx4 *)(part + row * LD + wj * (EDGE / 2) + 16 * j + 4 * (lane >> 4)) = acc[i][j];
            }
            __syncthreads();
            if (group == 0)
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    const int row = wi * (EDGE / 2) + 16 * i + (lane & 15);
                    if (sums && lane < 16) row_sum[i][0] += part_rows[row];
#pragma unroll
                    for (int j = 0; j < NB; ++j) acc[i][j] += *(const floatx4 *)(part + row * LD + wj * (EDGE / 2) + 16 * j + 4 * (lane >> 4));
                }
        }
    }
    if (PIECES && slot >= 0) {
        if (group > 0) return;
        float *const out = a.partial + slot * slot_floats<EDGE, EDGE>();
#pragma unroll
        for (int i = 0; i < NB; ++i) {
#pragma unroll
            for (int j = 0; j < NB; ++j) *(floatx4 *)(out + 4 * ((i * NB + j) * 256 + tid)) = acc[i][j];
            if (sums && lane < 16) out[EDGE * EDGE + wi * (EDGE / 2) + 16 * i + lane] = row_sum[i][0];
        }
        return;
    }
    // lane -> row lane % 16 of a block, columns 4 (lane / 16) .. + 3
    constexpr bool SAME = OP == EXPERT_FORWARD || OP == EXPERT_GRAD_INPUT;   // results of the operands' type
    constexpr int PART = EDGE == 128 && (FP32 || (sizeof(T) == 2 && !SAME)) ? 32 : 64;
    static_assert(PART * (EDGE + 8) * (SAME ? sizeof(T) : 4) <= sizeof(lds), "the part has to fit");
    store_rows<T, OP, EDGE, EDGE, PART, 256 * GROUPS>(a, t, lds, threadIdx.x, [&](int p0, auto put_quad) {
        if (group > 0) return;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int row = wi * (EDGE / 2) + 16 * i;
            if (row < p0 || row >= p0 + PART) continue;
#pragma unroll
            for (int j = 0; j < NB; ++j) put_quad(row + (lane & 15), wj * (EDGE / 2) + 16 * j + 4 * (lane >> 4), acc[i][j]);
        }
    });
    if (sums && group == 0 && lane < 16)
#pragma unroll
        for (int i = 0; i < NB; ++i) store_sum<OP>(a, t, t.ti * EDGE + wi * (EDGE / 2) + 16 * i + lane, row_sum[i][0]);
}

// ---- bf16, rows of whole 16-byte chunks: operands straight to LDS --------------------------------------
// BM x BN tiles, WI x WJ waves, in halves of 32 k.  Five halves have a place in LDS: while one is multiplied from registers and the
// fragments of the next one are read, the three behind it are there or on their way.  Loads go out for two halves (64 k, whole
// 128-byte lines of operands along k; half lines were fetched twice: 640 us for the forward product below) at a time and have three
// halves' time to arrive.
// 65536 rows 2048 -> 2048 of 16 experts: 540, 525 and 550 us for the three products, 1.0 PFLOP/s; 8192 rows 8192 -> 8192: 1.1 - 1.28 (the
// library's product has 1.41).  Bound by what the loads cost inside a CU and by power: without loads in the loop 375, 365 and
// 330 us, with loads of the same lines over and over 460, 451 and 541, at a shader clock of 1.64 - 1.8 GHz.  Four waves of
// 128 x 128, which read a quarter less from LDS, were slower (576, 562 and 664 us), as were two stages of 64 k (8192 rows: 1131, 1048
// and 918 us instead of 1006, 856 and 972).
// Offsets in a tensor are 32 bits (the host sees to it); rows and columns beyond the tile's are clamped, they reach no output.
// What is left of a contraction that is no whole number of steps of 64 goes through registers, with zeros behind its end.
constexpr int kPlaces = 5;
typedef float floatx16 __attribute__((ext_vector_type(16)));

// Which pairs of chunks of line m change places, so that the lanes of a transposing read meet different banks.
template <int ROWS>
__device__ __forceinline__ int swap_pairs(int m) { return ROWS == 64 ? m & 2 : (m & 3) << 1; }

// The 32 rows from `row0` (a multiple of 32) of a half, k = 16 u + 8 (lane / 32) .. + 7: lane -> row lane % 32.
template <bool ACROSS, int ROWS>
__device__ __forceinline__ bf16x8 fragment32(const bf16_t *tile, int row0, int u, int lane)
{
    if constexpr (ACROSS) {
        const int m = 16 * u + 8 * (lane >> 5) + ((lane & 15) >> 2), pair = (row0 >> 4) + ((lane >> 4) & 1);
        const bf16_t *p = tile + m * ROWS + 16 * (pair ^ swap_pairs<ROWS>(m)) + 4 * (lane & 3);
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_ptr)p);
        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_ptr)(p + 4 * ROWS));   // k + 4: same permutation
        return __builtin_bit_cast(bf16x8, shortx8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    } else {
        const int line = row0 + (lane & 31);
        return *(const bf16x8 *)(tile + 32 * line + 8 * ((2 * u + (lane >> 5)) ^ ((line >> 1) & 3)));
    }
}
__device__ __forceinline__ floatx16 mfma32(const bf16x8 &j, const bf16x8 &i, const floatx16 &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(j, i, c, 0, 0, 0);
}

// c and the two bf16 values of a register, in fp32: one instruction instead of four (factors of 32768 rows in 16 experts 75.4 -> 73.2 us);
// its roundings stay below 3 x 2^-24 of the largest, and sums of 4096 values in a row were off by as much as one by one.
__device__ __forceinline__ float add_pair(unsigned pair, float c)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3F803F80u), c, false);
}

template <bool ACROSS, int GATHER, int ROWS, int THREADS>
struct Direct {
    static constexpr int CH = ROWS * 4 / THREADS, PER = ACROSS ? ROWS / 8 : 4;   // chunks a thread and half, chunks a line
    static constexpr int LINES = 64 / PER;                               // (across k) lines that one load of a wave covers
    typedef const int __attribute__((address_space(4))) *order_ptr;      // read with scalar loads
    const char *base;
    unsigned off[CH];
    unsigned ld;      // bytes
    int begin, K, fan;
    unsigned magic;   // c / fan = (c * magic) >> 32
    int next[ACROSS && GATHER != 0 ? 2 * CH * LINES : 1];   // choices of the step that is loaded next

    __device__ __forceinline__ unsigned row_of(int c) const { return GATHER == 2 && fan > 1 ? __umulhi((unsigned)c, magic) : (unsigned)c; }
    __device__ __forceinline__ int choice(const ExpertArgs &a, int r) const   // always inside the tensor
    {
        return a.order ? min(max(a.order[begin + r], 0), a.n - 1) : begin + r;
    }
    __device__ __forceinline__ void fetch_choices(const ExpertArgs &a, int step, int wave)
    {
        if constexpr (ACROSS && GATHER != 0) {
            const order_ptr order = (order_ptr)(unsigned long long)a.order;
#pragma unroll
            for (int i = 0; i < 2 * CH; ++i)
#pragma unroll
                for (int q = 0; q < LINES; ++q) {
                    const int r = begin + min(64 * step + 32 * (i & 1) + (wave + THREADS / 64 * (i >> 1)) * LINES + q, K - 1);
                    next[i * LINES + q] = a.order ? order[r] : r;
                }
        }
    }
    __device__ __forceinline__ void init(const ExpertArgs &a, const void *base_, long long ld_, int fan_, int begin_, int row0, int rows, int K_, int tid)
    {
        base = (const char *)base_; ld = (unsigned)(2 * ld_); begin = begin_; K = K_; fan = fan_;
        magic = fan > 1 ? (unsigned)((0x100000000ULL + fan - 1) / fan) : 0;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int q = tid + THREADS * i, line = q / PER, phys = q % PER;
            if constexpr (ACROSS) {
                const int pos = (((phys >> 1) ^ swap_pairs<ROWS>(line)) << 1) | (phys & 1);
                off[i] = 2u * (unsigned)min(row0 + 8 * pos, rows - 8) + (GATHER == 0 ? (unsigned)line * ld : 0u);
            } else {
                int r = min(row0 + line, rows - 1);
                if constexpr (GATHER != 0) r = (int)row_of(choice(a, r));
                off[i] = (unsigned)r * ld + 16u * (unsigned)(phys ^ ((line >> 1) & 3));
            }
        }
    }
    __device__ __forceinline__ const char *half_base(int step, int u) const
    {
        if constexpr (!ACROSS) return base + 128LL * step + 64 * u;
        else if constexpr (GATHER == 0) return base + (64LL * step + 32 * u) * ld;
        else return base;
    }
    // load i of the thread's 2 CH of a step: chunk i / 2 of half i % 2, into the tile of that half
    __device__ __forceinline__ void load(const ExpertArgs &a, lds_address tile, int step, int i, int tid, int wave) const
    {
        unsigned o = off[i >> 1];
        if constexpr (ACROSS && GATHER != 0) {
            unsigned r = 0;
#pragma unroll
            for (int q = 0; q < LINES; ++q) {
                const unsigned at = row_of(min(max(next[i * LINES + q], 0), a.n - 1)) * ld;
                r = q == 0 || ((tid & 63) / PER) >= q ? at : r;
            }
            o += r;
        }
        load_to_lds(half_base(step, i & 1), o, tile + 16 * (64 * wave + THREADS * (i >> 1)));
    }
    // half u of the last, partial step
    __device__ __forceinline__ void load_rest(const ExpertArgs &a, bf16_t *tile, int step, int u, int tid) const
    {
        const char *from = half_base(step, u);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int line = (tid + THREADS * i) / PER;
            const int k = 64 * step + 32 * u + (ACROSS ? line : 8 * ((tid % PER) ^ ((line >> 1) & 3)));
            uintx4 v = {0, 0, 0, 0};
            if (k < K) {
                unsigned o = off[i];
                if constexpr (ACROSS && GATHER != 0) o += row_of(choice(a, k)) * ld;
                v = *(const uintx4 *)(from + o);
            }
            *(uintx4 *)(tile + 8 * (tid + THREADS * i)) = v;
        }
    }
};

template <int OP, int BM, int BN, int WI, int WJ, bool SUMS, bool PIECES>
__global__ __launch_bounds__(64 * WI * WJ, 2) void expert_direct_kernel(const ExpertArgs a, int tiles_j, int total)
{
    constexpr bool ACROSS_A = OP == EXPERT_GRAD_WEIGHT || OP == EXPERT_STATS;
    constexpr bool ACROSS_B = OP != EXPERT_FORWARD;
    constexpr int GATHER_X = PIECES ? 0 : 2;
    constexpr int GATHER_A = OP == EXPERT_FORWARD ? 2 : OP == EXPERT_STATS ? GATHER_X : 1;
    constexpr int GATHER_B = OP == EXPERT_GRAD_WEIGHT || OP == EXPERT_STATS ? GATHER_X : 0;
    constexpr int THREADS = 64 * WI * WJ, TI = BM / WI, TJ = BN / WJ, NI = TI / 32, NJ = TJ / 32, PLACE = (BM + BN) * 32;
    __shared__ __attribute__((aligned(1024))) bf16_t lds[kPlaces * PLACE];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave / WJ, wj = wave % WJ;
    Tile t;
    int slot = -1;
    if constexpr (PIECES) {
        if (!find_piece<OP, BM, BN>(a, tiles_j, total, t, slot)) return;
    } else {
        if (!find_work<OP, BM, BN>(a, tiles_j, total, t)) return;
    }

    typedef Direct<ACROSS_A, GATHER_A, BM, THREADS> DirectA;
    typedef Direct<ACROSS_B, GATHER_B, BN, THREADS> DirectB;
    constexpr int LA = 2 * DirectA::CH, LOADS = LA + 2 * DirectB::CH;   // a thread's, a step
    DirectA da;
    DirectB db;
    const bf16_t *We = (const bf16_t *)a.W + (long long)min(t.e, a.experts - 1) * a.co * a.ldw, *x = (const bf16_t *)a.x + (PIECES ? t.begin * a.ldx : 0);
    if constexpr (OP == EXPERT_FORWARD) da.init(a, x, a.ldx, a.fan, t.begin, t.ti * BM, t.I, t.K, tid);
    else if constexpr (OP == EXPERT_STATS) da.init(a, t.g ? (const bf16_t *)a.dy : x, t.g ? a.ldy : a.ldx, t.g ? 1 : a.fan, t.begin, t.ti * BM, t.I, t.K, tid);
    else da.init(a, a.dy, a.ldy, 1, t.begin, t.ti * BM, t.I, t.K, tid);
    if constexpr (OP == EXPERT_FORWARD || OP == EXPERT_GRAD_INPUT) db.init(a, We, a.ldw, 1, 0, t.tj * BN, t.J, t.K, tid);
    else if constexpr (OP == EXPERT_STATS) db.init(a, t.g ? (const bf16_t *)a.dy : x, t.g ? a.ldy : a.ldx, t.g ? 1 : a.fan, t.begin, t.tj * BN, t.J, t.K, tid);
    else db.init(a, x, a.ldx, a.fan, t.begin, t.tj * BN, t.J, t.K, tid);
    const bool sums = SUMS && wants_sums<OP>(a, t, wj);

    floatx16 acc[NI][NJ];
    float row_sum[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        row_sum[i] = 0.f;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    }
    const lds_address lds0 = address_in_lds(lds);
    auto load = [&](int s, int place, int q) {   // place: of the step's first half
        const int at = place + (q & 1) < kPlaces ? place + (q & 1) : place + (q & 1) - kPlaces;
        if (q < LA) da.load(a, lds0 + at * (2 * PLACE), s, q, tid, wave);
        else db.load(a, lds0 + at * (2 * PLACE) + BM * 64, s, q - LA, tid, wave);
    };
    auto fetch = [&](int s) {
        da.fetch_choices(a, s, wave);
        db.fetch_choices(a, s, wave);
    };
    // fragment q of a half: first those of its first 16 k
    auto read = [&](int place, int q, bf16x8 (&x)[2][NI], bf16x8 (&y)[2][NJ]) {
        const bf16_t *half = lds + place * PLACE;
        const int u = q / (NI + NJ), n = q % (NI + NJ);
        if (n < NI) x[u][n] = fragment32<ACROSS_A, BM>(half, wi * TI + 32 * n, u, lane);
        else y[u][n - NI] = fragment32<ACROSS_B, BN>(half + BM * 32, wj * TJ + 32 * (n - NI), u, lane);
    };
    auto multiply = [&](const bf16x8 (&x)[2][NI], const bf16x8 (&y)[2][NJ], int m) {
        const int u = m / (NI * NJ), j = m / NI % NJ, i = m % NI;
        acc[i][j] = mfma32(y[u][j], x[u][i], acc[i][j]);
    };
    auto add_rows = [&](const bf16x8 (&x)[2][NI]) {
        if constexpr (SUMS)
            if (sums)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
                        if constexpr (PIECES) {
                            const uintx4 pairs = __builtin_bit_cast(uintx4, x[u][i]);
#pragma unroll
                            for (int q = 0; q < 4; ++q) row_sum[i] = add_pair(pairs[q], row_sum[i]);
                        } else {
#pragma unroll
                            for (int q = 0; q < 8; ++q) row_sum[i] += (float)x[u][i][q];
                        }
                    }
    };
    const int whole = t.K / 64;
    if (whole > 0) {
        bf16x8 fa[2][2][NI], fb[2][2][NJ];   // [half][first or second 16 k]
        int place = 0;   // of the first half of the step that is multiplied
        auto behind = [&](int n) { return place + n < kPlaces ? place + n : place + n - kPlaces; };
        fetch(0);
#pragma unroll
        for (int q = 0; q < LOADS; ++q) load(0, 0, q);
        fetch(1);
        if (whole > 1) {
#pragma unroll
            for (int q = 0; q < LOADS; ++q) load(1, 2, q);
            fetch(2);
            wait_loads<LOADS>();
        } else {
            wait_loads<0>();
        }
#pragma unroll
        for (int q = 0; q < 2 * (NI + NJ); ++q) read(0, q, fa[0], fb[0]);
        // One half of a step: x y is multiplied; the fragments of the next half are read from `from`, and the loads of step s + 2 are
        // started if there is one, an access behind every few matrix instructions, which run meanwhile.
        auto half = [&](const bf16x8 (&x)[2][NI], const bf16x8 (&y)[2][NJ], int from, bf16x8 (&nx)[2][NI], bf16x8 (&ny)[2][NJ], auto first, bool more, int s,
                        int to) {
            constexpr int MM = 2 * NI * NJ, NR = 2 * (NI + NJ);
#pragma unroll
            for (int m = 0; m < MM; ++m) {
                multiply(x, y, m);
                // the reads end some instructions before the barrier
#pragma unroll
                for (int q = min(NR, NR * m / (MM * 3 / 4)); q < min(NR, NR * (m + 1) / (MM * 3 / 4)); ++q) read(from, q, nx, ny);
                if constexpr (first)
                    if (more)
#pragma unroll
                        for (int q = LOADS * m / MM; q < LOADS * (m + 1) / MM; ++q) load(s + 2, to, q);
                __builtin_amdgcn_sched_barrier(0);
            }
            add_rows(x);
        };
        for (int s = 0; s < whole; ++s) {
            const bool more = s + 2 < whole;
            wait_lds();   // everyone has read the first half of step s: its place and the one before it are free
            half(fa[0], fb[0], behind(1), fa[1], fb[1], std::true_type{}, more, s, behind(4));
            if (!PIECES) fetch(s + 3);
            if (more) wait_loads<LOADS>();   // step s + 1 is there
            else wait_loads<0>();
            if (PIECES) fetch(s + 3);        // (the wait is for scalar loads, too: these have half a step)
            half(fa[1], fb[1], behind(2), fa[0], fb[0], std::false_type{}, false, s, 0);   // (what is read behind the last step is not used)
            place = behind(2);
        }
        __syncthreads();   // everyone has read the last step
    }
    if (t.K > 64 * whole) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            da.load_rest(a, lds + u * PLACE, whole, u, tid);
            db.load_rest(a, lds + u * PLACE + BM * 32, whole, u, tid);
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            bf16x8 x[2][NI], y[2][NJ];
#pragma unroll
            for (int q = 0; q < 2 * (NI + NJ); ++q) read(u, q, x, y);
#pragma unroll
            for (int m = 0; m < 2 * NI * NJ; ++m) multiply(x, y, m);
            add_rows(x);
        }
    }
    if constexpr (SUMS)
#pragma unroll
        for (int i = 0; i < NI; ++i) row_sum[i] += __shfl_xor(row_sum[i], 32);   // the other 8 of 16 k
    if (PIECES && slot >= 0) {
        float *const out = a.partial + slot * slot_floats<BM, BN>();
#pragma unroll
        for (int i = 0; i < NI; ++i) {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *(floatx4 *)(out + 4 * (((i * NJ + j) * 4 + g) * THREADS + tid)) =
                        floatx4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
            if (sums && lane < 32) out[BM * BN + wi * TI + 32 * i + lane] = row_sum[i];
        }
        return;
    }
    // lane -> row lane % 32 of a block, columns 8 g + 4 (lane / 32) .. + 3 for its 16 sums in fours
    constexpr int SIZE = OP == EXPERT_FORWARD || OP == EXPERT_GRAD_INPUT ? 2 : 4;
    constexpr int PART = BM * (BN + 8) * SIZE <= (int)sizeof(lds) ? BM : BM / 2;
    static_assert(PART * (BN + 8) * SIZE <= sizeof(lds), "the part has to fit");
    store_rows<bf16_t, OP, BM, BN, PART, THREADS>(a, t, lds, tid, [&](int p0, auto put_quad) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int row = wi * TI + 32 * i;
            if (row < p0 || row >= p0 + PART) continue;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    put_quad(row + (lane & 31), wj * TJ + 32 * j + 8 * g + 4 * (lane >> 5),
                             floatx4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]});
        }
    });
    if (sums && lane < 32)
#pragma unroll
        for (int i = 0; i < NI; ++i) store_sum<OP>(a, t, t.ti * BM + wi * TI + 32 * i + lane, row_sum[i]);
}

// ---- the pieces' sums together ---------------------------------------------------------------------------
// Experts with several pieces: a thread adds up four times four adjacent sums of a tile over the pieces, in their order, and stores them as the
// kernels do.  Bound by memory: 16 factors of 1025 x 1025 from pieces 12 us.
template <int OP, bool DIRECT, int BM, int BN, int WI, int WJ>
__global__ __launch_bounds__(256) void expert_join_kernel(const ExpertArgs a, int tiles_j, int tiles)
{
    constexpr int QUADS = 4, PARTS = BM * BN / (1024 * QUADS), THREADS = 64 * WI * WJ, TI = BM / WI, TJ = BN / WJ;   // QUADS a thread
    const Pieces p = pieces_of<OP>(a);
    const int of = blockIdx.x / (tiles * PARTS), rest = blockIdx.x - of * tiles * PARTS, local = rest / PARTS, part = rest - local * PARTS;
    const unsigned long long has = __ballot(p.count > 1 && p.split == of);
    if (!has) return;
    Tile t;
    t.e = __ffsll(has) - 1;
    t.len = __builtin_amdgcn_readlane(p.len, t.e);
    const int count = __builtin_amdgcn_readlane(p.count, t.e), place = __builtin_amdgcn_readlane(p.slot, t.e);
    if (place + count > a.most) return;
    row_tile<OP, BM, BN>(a, tiles_j, local, t);
    const float *from = a.partial + ((long long)place * tiles + local) * slot_floats<BM, BN>();
    const long long apart = tiles * slot_floats<BM, BN>();
    floatx4 sum[QUADS];
#pragma unroll
    for (int u = 0; u < QUADS; ++u) sum[u] = *(const floatx4 *)(from + 4 * ((part * QUADS + u) * 256 + threadIdx.x));
    for (int k = 1; k < count; ++k)
#pragma unroll
        for (int u = 0; u < QUADS; ++u) sum[u] += *(const floatx4 *)(from + k * apart + 4 * ((part * QUADS + u) * 256 + threadIdx.x));
#pragma unroll
    for (int u = 0; u < QUADS; ++u) {
        const int quad = (part * QUADS + u) * 256 + threadIdx.x, q = quad / THREADS, tid = quad % THREADS, lane = tid & 63, wi = (tid >> 6) / WJ, wj = (tid >> 6) % WJ;
        int row, col;
        if constexpr (DIRECT) {
            constexpr int NJ = TJ / 32;
            row = wi * TI + 32 * (q / 4 / NJ) + (lane & 31);
            col = wj * TJ + 32 * (q / 4 % NJ) + 8 * (q % 4) + 4 * (lane >> 5);
        } else {
            constexpr int NJ = TJ / 16;
            row = wi * TI + 16 * (q / NJ) + (lane & 15);
            col = wj * TJ + 16 * (q % NJ) + 4 * (lane >> 4);
        }
        row += t.ti * BM;
        col += t.tj * BN;
        if (row >= t.I) continue;
        if constexpr (OP == EXPERT_GRAD_WEIGHT) {
            store4<float>(a.dW + ((long long)t.e * a.co + row) * (a.ci + a.bias) + col, t.J - col, sum[u]);
        } else {
            const int d = a.ci + a.bias, below = min(row + 1 - col, 4);   // the lower triangle and its mirror image
            float *const M = a.A + (long long)t.e * d * d, *const out = M + (long long)row * d + col;
            const float alpha = (1.f - a.decay) / (float)t.len;
            floatx4 v;
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = blend(a.decay, alpha, a.decay != 0.f && r < below ? out[r] : 0.f, sum[u][r]);
            store4<float>(out, below, v);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r < below && col + r < row) M[(long long)(col + r) * d + row] = v[r];
        }
    }
    if (a.bias && t.tj == 0 && part == 0 && threadIdx.x < BM) {
        float sum = 0.f;
        for (int k = 0; k < count; ++k) sum += from[k * apart + BM * BN + threadIdx.x];
        store_sum<OP>(a, t, t.ti * BM + (int)threadIdx.x, sum);
    }
}

// Operands that go straight to LDS: whole 16-byte chunks, offsets of 32 bits, choices that the division by `fan` is exact for.
bool chunks(const void *p, long long rows, long long cols, long long ld)
{
    return ((uintptr_t)p % 16) == 0 && ld % 8 == 0 && cols % 8 == 0 && cols >= 8 && rows * ld < (1LL << 31);
}
bool direct_ok(ExpertOp op, const ExpertArgs &a)
{
    if ((long long)a.n * a.fan >= (1LL << 32)) return false;
    const bool x = chunks(a.x, a.n / a.fan, a.ci, a.ldx), dy = chunks(a.dy, a.n, a.co, a.ldy);
    switch (op) {
        case EXPERT_FORWARD: return x && chunks(a.W, a.co, a.ci, a.ldw);
        case EXPERT_GRAD_INPUT: return dy && chunks(a.W, a.co, a.ci, a.ldw);
        case EXPERT_GRAD_WEIGHT: return x && dy;
        case EXPERT_STATS: return (!a.A || x) && (!a.G || dy);
    }
    return false;
}

template <int BM, int BN>
long long count_tiles(ExpertOp op, const ExpertArgs &a, int &tiles_j)
{
    tiles_j = 1;
    if (op == EXPERT_FORWARD || op == EXPERT_GRAD_INPUT) {   // at most: one ragged tile a segment
        tiles_j = ((op == EXPERT_FORWARD ? a.co : a.ci) + BN - 1) / BN;
        return (long long)(a.n / BM + (a.n < a.experts + 1 ? a.n : a.experts + 1)) * tiles_j;
    }
    if (op == EXPERT_GRAD_WEIGHT) {
        tiles_j = (a.ci + BN - 1) / BN;
        return (long long)a.experts * (((long long)((a.co + BM - 1) / BM) * tiles_j + 7) / 8 * 8);
    }
    return (long long)a.experts * (((a.A ? triangle_tiles<BM>(a.ci) : 0) + (a.G ? triangle_tiles<BM>(a.co) : 0) + 7) / 8 * 8);
}

template <int BM, int BN, int WI, int WJ>
hipError_t run_direct(ExpertOp op, const ExpertArgs &a, hipStream_t s)
{
    int tj;
    const long long wgs = count_tiles<BM, BN>(op, a, tj);
    const dim3 grid((unsigned)wgs), block(64 * WI * WJ);
    switch (op) {
        case EXPERT_FORWARD: expert_direct_kernel<EXPERT_FORWARD, BM, BN, WI, WJ, false, false><<<grid, block, 0, s>>>(a, tj, (int)wgs); break;
        case EXPERT_GRAD_INPUT: expert_direct_kernel<EXPERT_GRAD_INPUT, BM, BN, WI, WJ, false, false><<<grid, block, 0, s>>>(a, tj, (int)wgs); break;
        default: return hipErrorInvalidValue;   // (run_direct_rows has the others)
    }
    return hipGetLastError();
}

// The contractions over rows
template <int BM, int BN, int WI, int WJ>
hipError_t run_direct_rows(ExpertOp op, const ExpertArgs &a, hipStream_t s)
{
    int tj;
    const long long wgs = count_tiles<BM, BN>(op, a, tj);
    const dim3 grid((unsigned)wgs), block(64 * WI * WJ);
    if (op == EXPERT_GRAD_WEIGHT) {
        if (a.bias) expert_direct_kernel<EXPERT_GRAD_WEIGHT, BM, BN, WI, WJ, true, false><<<grid, block, 0, s>>>(a, tj, (int)wgs);
        else expert_direct_kernel<EXPERT_GRAD_WEIGHT, BM, BN, WI, WJ, false, false><<<grid, block, 0, s>>>(a, tj, (int)wgs);
    } else {
        if (a.bias) expert_direct_kernel<EXPERT_STATS, BM, BN, WI, WJ, true, false><<<grid, block, 0, s>>>(a, tj, (int)wgs);
        else expert_direct_kernel<EXPERT_STATS, BM, BN, WI, WJ, false, false><<<grid, block, 0, s>>>(a, tj, (int)wgs);
    }
    return hipGetLastError();
}

template <typename T, bool FP32, ExpertOp OP, int EDGE, int GROUPS>
hipError_t run_general(const ExpertArgs &a, hipStream_t s)
{
    int tj;
    const long long wgs = count_tiles<EDGE, EDGE>(OP, a, tj);
    expert_general_kernel<T, FP32, OP, EDGE, GROUPS, false><<<dim3((unsigned)wgs), dim3(256 * GROUPS), 0, s>>>(a, tj, (int)wgs);
    return hipGetLastError();
}

// 128 x 128 tiles where there are two for each CU, smaller ones otherwise: fp32 2051 rows 515 -> 1000 of 8 uneven experts take 47, 88 and
// 141 us for the three products with the large ones (200, 125 and 320 tiles), 32, 49 and 66 with the small ones and one group, 36, 38 and
// 46 with two.  Even experts, small with two groups and large: forward 135 and 150 us at 657 large tiles, 249 and 230 at 1241; weights 21.5
// and 21.8 at 512, 88 and 112 at 640, 55 and 53 at 1408; factors 27 and 28 at 512, 117 and 130 at 896.
// Contractions over rows of few tiles are chains as long as the longest expert: four groups up to 512 small tiles.  Uneven experts, fp32
// factors of 2053 rows, 448 tiles: 55, 36 and 27 us with one, two and four; of 2048 rows, 1376 tiles: 42 with two, 59 with four.  Even
// experts, four and two: weights 15 and 20 us at 64 tiles, 11 and 13 at 256, 19 and 15.5 at 512, 32 and 25 at 832.
template <typename T, bool FP32, ExpertOp OP>
hipError_t general(const ExpertArgs &a, hipStream_t s)
{
    int tj;
    if (count_tiles<128, 128>(OP, a, tj) >= 512) return run_general<T, FP32, OP, 128, 1>(a, s);
    if constexpr (OP == EXPERT_GRAD_WEIGHT || OP == EXPERT_STATS)
        if (count_tiles<64, 64>(OP, a, tj) <= 512) return run_general<T, FP32, OP, 64, 4>(a, s);
    return run_general<T, FP32, OP, 64, 2>(a, s);
}

template <typename T, bool FP32>
hipError_t general(ExpertOp op, const ExpertArgs &a, hipStream_t s)
{
    switch (op) {
        case EXPERT_FORWARD: return general<T, FP32, EXPERT_FORWARD>(a, s);
        case EXPERT_GRAD_INPUT: return general<T, FP32, EXPERT_GRAD_INPUT>(a, s);
        case EXPERT_GRAD_WEIGHT: return general<T, FP32, EXPERT_GRAD_WEIGHT>(a, s);
        case EXPERT_STATS: return general<T, FP32, EXPERT_STATS>(a, s);
    }
    return hipErrorInvalidValue;
}

// ---- contractions over rows in pieces -------------------------------------------------------------------
// Every CU shall have work and the pieces shall be few (their sums go to memory and back): as many rows as a tile has if all of them went
// evenly to `slots` workgroups, 512 at least, and more if the sums had no room.  128 x 128, two a CU, 512 slots: factors of 32768 rows 1024
// channels in one expert 82 us, in 16 uneven ones 108 (384: 96 and 110, 768: 82 and 113, 1024: 85 and 120); of the same in tiles of 256 x 256
// 99 and 117.
int most_pieces(long long n, int experts, int piece) { return (int)std::min(2 * n / piece, n / piece + experts); }   // of experts with several: each is longer than half a piece
int piece_rows(long long n, int experts, int tiles, int slots, size_t slot_bytes, size_t room)
{
    const long long even = std::min((n * tiles + slots - 1) / slots, n);
    long long rows = std::max(512LL, (even + 63) / 64 * 64);
    while (rows < n && (size_t)most_pieces(n, experts, (int)rows) * tiles * slot_bytes > room) rows += std::max(64LL, rows / 16 / 64 * 64);
    return (int)rows;
}
template <int OP, int BM, int BN>
int row_tiles(const ExpertArgs &a, int &tiles_j)
{
    tiles_j = (a.ci + BN - 1) / BN;
    if (OP == EXPERT_GRAD_WEIGHT) return (a.co + BM - 1) / BM * tiles_j;
    return triangle_tiles<BM>(a.ci);
}

template <ExpertOp OP, bool DIRECT, int BM, int BN, int WI, int WJ, typename Launch>
hipError_t run_pieces(ExpertArgs a, int slots, hipStream_t s, Launch launch)
{
    int tj;
    const int tiles = row_tiles<OP, BM, BN>(a, tj);
    a.piece = piece_rows(a.n, a.experts, tiles, slots, slot_floats<BM, BN>() * sizeof(float), expert_pieces_bytes(a.experts, a.n, a.ci, a.co));
    a.most = a.n > a.piece ? most_pieces(a.n, a.experts, a.piece) : 0;
    a.whole_pieces = BM < 256 && tiles <= slots / 8;   // then there are eight pieces at least (dense factors above: 101 us in eighths; weights in tiles of 256: 134 whole, 116)
    const int most = a.n / a.piece + a.experts;
    launch(a, dim3((unsigned)(a.whole_pieces ? (most + 7) / 8 * 8 * tiles : most * ((tiles + 7) / 8 * 8))), tj, tiles);
    if (a.n > a.piece)   // at most n / piece experts have several
        expert_join_kernel<OP, DIRECT, BM, BN, WI, WJ><<<dim3((unsigned)(a.n / a.piece) * tiles * (BM * BN / 4096)), dim3(256), 0, s>>>(a, tj, tiles);
    return hipGetLastError();
}

template <ExpertOp OP, int BM, int BN, int WI, int WJ>
hipError_t run_direct_pieces(const ExpertArgs &a, int slots, hipStream_t s)
{
    return run_pieces<OP, true, BM, BN, WI, WJ>(a, slots, s, [&](const ExpertArgs &p, dim3 grid, int tj, int tiles) {
        if (p.bias) expert_direct_kernel<OP, BM, BN, WI, WJ, true, true><<<grid, dim3(64 * WI * WJ), 0, s>>>(p, tj, tiles);
        else expert_direct_kernel<OP, BM, BN, WI, WJ, false, true><<<grid, dim3(64 * WI * WJ), 0, s>>>(p, tj, tiles);
    });
}
template <typename T, bool FP32, ExpertOp OP, int EDGE, int GROUPS>
hipError_t run_general_pieces(const ExpertArgs &a, int slots, hipStream_t s)
{
    return run_pieces<OP, false, EDGE, EDGE, 2, 2>(a, slots, s, [&](const ExpertArgs &p, dim3 grid, int tj, int tiles) {
        expert_general_kernel<T, FP32, OP, EDGE, GROUPS, true><<<grid, dim3(256 * GROUPS), 0, s>>>(p, tj, tiles);
    });
}

template <ExpertOp OP>
hipError_t pieces(const ExpertArgs &a, bool bf16, bool planes, hipStream_t s)
{
    int tj;
    if (bf16 && direct_ok(OP, a)) {
        // 256 x 256, one a CU, needs long contractions for what it does not overlap: with 2048 rows for each CU on (weights 1024 -> 2048 of 16384 rows
        // in one expert 89 us, 109 with 128 x 128; in 16 uneven ones 116 and 154)
        if ((long long)a.n * row_tiles<OP, 256, 256>(a, tj) >= 2048 * 256) return run_direct_pieces<OP, 256, 256, 4, 2>(a, 256, s);
        return run_direct_pieces<OP, 128, 128, 2, 2>(a, 512, s);
    }
    // 128 x 128 where the experts have 512 such tiles, 64 x 64 with two groups of waves below.  Weights in fp32, large and small: 477 and 640 us at
    // 2048 tiles (8192 rows, two choices each), 156 and 179 at 512 (4096 rows), but 59 and 77 at 256 (2048 rows) and 392 and 545 for one expert
    // with 128 (16384 rows), where the small ones are taken; bf16, no row aligned: 304 and 350 at 2048, 113 and 110 at 512, 365 and 434 for one
    // expert with 128.  Factors in fp32: 258 and 274 at 576, 96 and 84 at 288, 48 and 41 at 80; bf16, no row aligned: 173 and 178 at 576, 71 and
    // 66 at 288.
    if (a.experts * row_tiles<OP, 128, 128>(a, tj) >= 512) {
        if (bf16) return run_general_pieces<bf16_t, false, OP, 128, 1>(a, 512, s);
        return planes ? run_general_pieces<float, false, OP, 128, 1>(a, 512, s) : run_general_pieces<float, true, OP, 128, 1>(a, 512, s);
    }
    if (bf16) return run_general_pieces<bf16_t, false, OP, 64, 2>(a, 1024, s);
    return planes ? run_general_pieces<float, false, OP, 64, 2>(a, 1024, s) : run_general_pieces<float, true, OP, 64, 2>(a, 1024, s);
}

}  // namespace

size_t expert_pieces_bytes(int experts, int n, int ci, int co)
{
    if (experts > 64) return 0;
    // room for n / 256 pieces or for about 64 MiB of them
    const size_t i = ((size_t)ci + 255) / 256 * 256, o = ((size_t)co + 255) / 256 * 256;
    const size_t piece = i * std::max(i, o) * sizeof(float) / 64 * 65, most = (size_t)1024 * (128 * 128 / 64 * 65) * sizeof(float);
    return std::min((size_t)(n / 256) * piece, most);
}

hipError_t launch_expert(ExpertOp op, const ExpertArgs &a, int bf16, bool planes, hipStream_t s)
{
    int tj;
    if (bf16 && direct_ok(op, a)) {
        // 256 x 256 tiles need half the traffic of 128 x 128, but one of them fills a CU: only where there is one for each of the 256
        // (16384 rows 1024 -> 2048 of 16 even experts, forward: 72 us, 83 with 128 x 128; uneven ones, whose last round is partial: 92 and
        // 86; 4096 rows 2048 -> 2048, 264 tiles: 54 and 56; 2048 rows 1024 -> 1024 of 8, 68 tiles: 28 and 17).  Weights of 16384 rows,
        // uneven: 113 and 103 us at 128 tiles, 69 and 78 at 256, 96 and 144 at 512; factors 137 and 136 at 192, 107 and 119 at 384, 218 and
        // 268 at 768.
        const bool full = count_tiles<256, 256>(op, a, tj) >= 256;
        if (op == EXPERT_GRAD_WEIGHT || op == EXPERT_STATS) return full ? run_direct_rows<256, 256, 4, 2>(op, a, s) : run_direct_rows<128, 128, 2, 2>(op, a, s);
        if (full) return run_direct<256, 256, 4, 2>(op, a, s);
        // few rows an expert: 64 x 64, more of them in flight (a decoding step of 8 choices 1024 -> 4096: 14 us, 17 with 128 x 128; 2048
        // rows 1024 -> 1024 of 8 experts: 13 and 17; 4096 of 16: 21 and 19).  Gradients of weights have as many tiles whatever the rows
        // (2048 rows of 8 experts: 29 us, 19 with 128 x 128).
        return count_tiles<128, 128>(op, a, tj) <= 320 ? run_direct<64, 64, 2, 2>(op, a, s) : run_direct<128, 128, 2, 2>(op, a, s);
    }
    if (bf16) return general<bf16_t, false>(op, a, s);
    return planes ? general<float, false>(op, a, s) : general<float, true>(op, a, s);
}

hipError_t launch_expert_pieces(ExpertOp op, const ExpertArgs &a, int bf16, bool planes, hipStream_t s)
{
    return op == EXPERT_GRAD_WEIGHT ? pieces<EXPERT_GRAD_WEIGHT>(a, bf16, planes, s) : pieces<EXPERT_STATS>(a, bf16, planes, s);
}

}  // namespace kfac
