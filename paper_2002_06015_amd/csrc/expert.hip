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
// m m, h l, l h), all accumulated in fp32.
#include "gemm_tiles.h"
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

// Tile `block` of those of all experts with BM rows and tiles_j columns of tiles each; false: there are fewer.  Consecutive
// tiles share a panel of W; every XCD works through one contiguous share.  All threads of a wave call it.
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
            const int rows = (len + BM - 1) / BM;
            const int local = id - before - (__builtin_amdgcn_readlane(incl, who) - __builtin_amdgcn_readlane(t, who));
            tj = local / rows;
            ti = local - tj * rows;
            return true;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
    }
    return false;
}

// ---- tiles in LDS --------------------------------------------------------------------------------------
// 16-byte chunks of 8 elements.  Along k: line = row of the tile, BK / 8 chunks; across k: line = k, 16 chunks of 8 rows.
// Chunks are permuted inside a line so that the lanes of a read meet different banks.
template <bool ACROSS, int BK>
__device__ __forceinline__ int chunk_at(int line, int pos)
{
    if constexpr (ACROSS) return line * 16 + ((((pos >> 1) ^ ((line & 3) | ((line >> 1) & 4))) << 1) | (pos & 1));
    else if constexpr (BK == 64) return line * 8 + (pos ^ (line & 7));
    else return line * 4 + (pos ^ ((line >> 1) & 3));
}

// The 16 rows from `row0` (a multiple of 16) of a tile, k = 32 u + 8 (lane / 16) .. + 7: lane -> row lane % 16.
template <bool ACROSS, int BK>
__device__ __forceinline__ bf16x8 fragment(const bf16_t *tile, int row0, int u, int lane)
{
    if constexpr (ACROSS) {
        const int m = 32 * u + 8 * (lane >> 4) + ((lane & 15) >> 2);
        const bf16_t *p = tile + 8 * chunk_at<true, BK>(m, row0 / 8) + 4 * (lane & 3);   // (the pair of chunks stays together)
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_ptr)p);
        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_ptr)(p + 4 * 128));   // k + 4: same permutation
        return __builtin_bit_cast(bf16x8, shortx8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    } else {
        return *(const bf16x8 *)(tile + 8 * chunk_at<false, BK>(row0 + (lane & 15), 4 * u + (lane >> 4)));
    }
}

// ---- general kernel: any size, stride and alignment -----------------------------------------------------
// 128 x 128 tiles, four waves of 64 x 64; operands go through registers (converted there if they are fp32) into one LDS
// stage while the next step's loads are in flight.
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
};

// One operand of a tile.  Along k: rows [0, rows) from `line`; across k: columns col0 .. of `cols`, k < K.
// GATHER: 0: line r is base + r ld;  1: base + choice_at(begin + r) ld;  2: base + choice_at(begin + r) / fan * ld
// (fan: 1 where the rows are those of the choices)
template <typename T, bool ACROSS, int GATHER, int BK>
struct Staged {
    static constexpr int CH = BK / 16, PER = ACROSS ? 16 : BK / 8;
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
    // rows: of the tile's first row on (along k); cols and K as above
    __device__ __forceinline__ void init(const ExpertArgs &a, const T *base_, long long ld_, int fan_, int begin_, int row0, int rows, int K_, int tid)
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
            next_choices(a, 0, tid);
        }
    }
    __device__ __forceinline__ void load(const ExpertArgs &a, int k0, int tid)
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
        if constexpr (ACROSS && GATHER != 0) next_choices(a, k0 + BK, tid);
    }
    __device__ __forceinline__ void store(bf16_t *tile, int tid) const
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int q = tid + 256 * i;
            reg[i].store(tile, 128 * BK, chunk_at<ACROSS, BK>(q / PER, q % PER));
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

// Which tile of which factor a workgroup of the statistics forms.
struct StatsTile {
    int e, begin, len, ti, tj, dim;
    bool g;
};

__device__ __forceinline__ bool find_stats_tile(const ExpertArgs &a, int block, int total, int edge, StatsTile &t)
{
    const int ta = a.A ? (a.ci + edge - 1) / edge : 0, tg = a.G ? (a.co + edge - 1) / edge : 0;
    const int na = ta * (ta + 1) / 2, per = na + tg * (tg + 1) / 2;
    const int id = xcd_remap(block, total);
    t.e = id / per;
    int local = id - t.e * per;
    t.g = local >= na;
    if (t.g) local -= na;
    tri_decode(local, t.ti, t.tj);
    t.dim = t.g ? a.co : a.ci;
    segment(a, t.e, t.begin, t.len);
    return t.len > 0;
}

template <typename T, int OP>
__global__ __launch_bounds__(256, 2) void expert_general_kernel(const ExpertArgs a, int tiles_j, int total)
{
    constexpr int BK = sizeof(T) == 2 ? 64 : 32, NP = sizeof(T) == 2 ? 1 : 3;
    constexpr bool ACROSS_A = OP == EXPERT_GRAD_WEIGHT || OP == EXPERT_STATS;
    constexpr bool ACROSS_B = OP != EXPERT_FORWARD;
    constexpr int GATHER_A = OP == EXPERT_FORWARD || OP == EXPERT_STATS ? 2 : 1;
    constexpr int GATHER_B = OP == EXPERT_GRAD_WEIGHT || OP == EXPERT_STATS ? 2 : 0;
    constexpr int PLANE = 128 * BK;
    __shared__ __attribute__((aligned(16))) bf16_t lds[2 * NP * PLANE];
    bf16_t *tile_a = lds, *tile_b = lds + NP * PLANE;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave >> 1, wj = wave & 1;

    int e, begin, len, ti, tj, I, J, K;
    bool sym_g = false;
    if constexpr (OP == EXPERT_FORWARD || OP == EXPERT_GRAD_INPUT) {
        if (!find_tile<128>(a, blockIdx.x, tiles_j, e, begin, len, ti, tj)) return;
        I = len;
        J = OP == EXPERT_FORWARD ? a.co : a.ci;
        K = e == a.experts ? 0 : OP == EXPERT_FORWARD ? a.ci : a.co;   // rows of choices that no expert takes are zero
    } else if constexpr (OP == EXPERT_GRAD_WEIGHT) {
        const int per = total / a.experts, id = xcd_remap(blockIdx.x, total);
        e = id / per;
        ti = (id - e * per) / tiles_j;
        tj = (id - e * per) - ti * tiles_j;
        segment(a, e, begin, len);
        I = a.co; J = a.ci; K = len;
    } else {
        StatsTile t;
        if (!find_stats_tile(a, blockIdx.x, total, 128, t)) return;
        e = t.e; begin = t.begin; len = t.len; ti = t.ti; tj = t.tj; sym_g = t.g;
        I = J = t.dim; K = len;
    }

    Staged<T, ACROSS_A, GATHER_A, BK> sa;
    Staged<T, ACROSS_B, GATHER_B, BK> sb;
    const T *We = (const T *)a.W + (long long)min(e, a.experts - 1) * a.co * a.ldw;
    if constexpr (OP == EXPERT_FORWARD) {
        sa.init(a, (const T *)a.x, a.ldx, a.fan, begin, ti * 128, I, K, tid);
        sb.init(a, We, a.ldw, 1, 0, tj * 128, J, K, tid);
    } else if constexpr (OP == EXPERT_GRAD_INPUT) {
        sa.init(a, (const T *)a.dy, a.ldy, 1, begin, ti * 128, I, K, tid);
        sb.init(a, We, a.ldw, 1, 0, tj * 128, J, K, tid);
    } else if constexpr (OP == EXPERT_GRAD_WEIGHT) {
        sa.init(a, (const T *)a.dy, a.ldy, 1, begin, ti * 128, I, K, tid);
        sb.init(a, (const T *)a.x, a.ldx, a.fan, begin, tj * 128, J, K, tid);
    } else {
        sa.init(a, (const T *)(sym_g ? a.dy : a.x), sym_g ? a.ldy : a.ldx, sym_g ? 1 : a.fan, begin, ti * 128, I, K, tid);
        sb.init(a, (const T *)(sym_g ? a.dy : a.x), sym_g ? a.ldy : a.ldx, sym_g ? 1 : a.fan, begin, tj * 128, J, K, tid);
    }
    // sums over k of the rows: the bias column of dW (with the tiles of the first columns), the border of A (with the diagonal)
    const bool sums = a.bias && ((OP == EXPERT_GRAD_WEIGHT && tj == 0) || (OP == EXPERT_STATS && !sym_g && ti == tj)) && wj == 0;
    bf16x8 ones;
#pragma unroll
    for (int q = 0; q < 8; ++q) ones[q] = (__bf16)1.f;

    floatx4 acc[4][4], row_sum[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        row_sum[i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    if (K > 0) {
        sa.load(a, 0, tid);
        sb.load(a, 0, tid);
    }
    for (int k0 = 0; k0 < K; k0 += BK) {
        if (k0 > 0) __syncthreads();   // every wave has read the step before
        sa.store(tile_a, tid);
        sb.store(tile_b, tid);
        __syncthreads();
        if (k0 + BK < K) {
            sa.load(a, k0 + BK, tid);
            sb.load(a, k0 + BK, tid);
        }
#pragma unroll
        for (int u = 0; u < BK / 32; ++u) {
            bf16x8 fa[NP][4], fb[NP][4];
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    fa[p][q] = fragment<ACROSS_A, BK>(tile_a + p * PLANE, wi * 64 + 16 * q, u, lane);
                    fb[p][q] = fragment<ACROSS_B, BK>(tile_b + p * PLANE, wj * 64 + 16 * q, u, lane);
                }
            constexpr int pa[6] = {0, 2, 1, 0, 1, 0}, pb[6] = {2, 0, 1, 1, 0, 0};   // the small products first
#pragma unroll
            for (int t = NP == 1 ? 5 : 0; t < 6; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = mfma(fb[pb[t]][j], fa[pa[t]][i], acc[i][j]);
            if (sums)
#pragma unroll
                for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                    for (int i = 0; i < 4; ++i) row_sum[i] = mfma(ones, fa[p][i], row_sum[i]);
        }
    }

    // lane -> row i = lane % 16 of a 16 x 16 block, columns 4 (lane / 16) .. + 3
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = ti * 128 + wi * 64 + 16 * i + (lane & 15);
        if (row >= I) continue;
        if constexpr (OP == EXPERT_FORWARD || OP == EXPERT_GRAD_INPUT) {
            const int c = choice_at(a, begin + row);
            if (c < 0) continue;
            T *out = (T *)a.out + (long long)c * a.ldo;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int col = tj * 128 + wj * 64 + 16 * j + 4 * (lane >> 4);
                floatx4 v = acc[i][j];
                if (OP == EXPERT_FORWARD && a.bias && e < a.experts)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (col + r < J) {
                            const T w = We[(long long)(col + r) * a.ldw + a.ci];
                            if constexpr (sizeof(T) == 2) v[r] += __uint_as_float((unsigned)w << 16);
                            else v[r] += w;
                        }
                store4<T>(out + col, J - col, v);
            }
        } else if constexpr (OP == EXPERT_GRAD_WEIGHT) {
            float *out = a.dW + ((long long)e * a.co + row) * (a.ci + a.bias);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int col = tj * 128 + wj * 64 + 16 * j + 4 * (lane >> 4);
                store4<float>(out + col, J - col, acc[i][j]);
            }
            if (sums && lane < 16) out[a.ci] = row_sum[i][0];
        } else {
            const int d = sym_g ? a.co : a.ci + a.bias;
            float *M = (sym_g ? a.G : a.A) + (long long)e * d * d;
            const float alpha = (1.f - a.decay) / (float)len;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int col = tj * 128 + wj * 64 + 16 * j + 4 * (lane >> 4) + r;
                    if (col > row) continue;               // (off the diagonal all columns are smaller)
                    float *lo = M + (long long)row * d + col;
                    const float v = blend(a.decay, alpha, a.decay == 0.f ? 0.f : *lo, acc[i][j][r]);
                    *lo = v;
                    if (col < row) M[(long long)col * d + row] = v;
                }
            if (sums && lane < 16) {
                float *lo = M + (long long)a.ci * d + row;
                const float v = blend(a.decay, alpha, a.decay == 0.f ? 0.f : *lo, row_sum[i][0]);
                *lo = v;
                M[(long long)row * d + a.ci] = v;
                if (row == 0) {
                    float *corner = M + (long long)a.ci * d + a.ci;
                    *corner = blend(a.decay, 1.f - a.decay, a.decay == 0.f ? 0.f : *corner, 1.f);
                }
            }
        }
    }
}

template <typename T>
hipError_t run(ExpertOp op, const ExpertArgs &a, hipStream_t s, int *workgroups)
{
    long long wgs = 0;
    int tj = 1;
    const long long tiles_n = a.n / 128 + (a.n < a.experts + 1 ? a.n : a.experts + 1);   // at most: one ragged tile a segment
    if (op == EXPERT_FORWARD || op == EXPERT_GRAD_INPUT) {
        tj = ((op == EXPERT_FORWARD ? a.co : a.ci) + 127) / 128;
        wgs = tiles_n * tj;
    } else if (op == EXPERT_GRAD_WEIGHT) {
        tj = (a.ci + 127) / 128;
        wgs = (long long)a.experts * ((a.co + 127) / 128) * tj;
    } else {
        const long long ta = a.A ? (a.ci + 127) / 128 : 0, tg = a.G ? (a.co + 127) / 128 : 0;
        wgs = a.experts * (ta * (ta + 1) / 2 + tg * (tg + 1) / 2);
    }
    if (wgs >= (1LL << 30)) return hipErrorInvalidValue;   // (refused by the entry points before)
    *workgroups = (int)wgs;
    const dim3 grid((unsigned)wgs), block(256);
    switch (op) {
        case EXPERT_FORWARD: expert_general_kernel<T, EXPERT_FORWARD><<<grid, block, 0, s>>>(a, tj, (int)wgs); break;
        case EXPERT_GRAD_INPUT: expert_general_kernel<T, EXPERT_GRAD_INPUT><<<grid, block, 0, s>>>(a, tj, (int)wgs); break;
        case EXPERT_GRAD_WEIGHT: expert_general_kernel<T, EXPERT_GRAD_WEIGHT><<<grid, block, 0, s>>>(a, tj, (int)wgs); break;
        case EXPERT_STATS: expert_general_kernel<T, EXPERT_STATS><<<grid, block, 0, s>>>(a, tj, (int)wgs); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_expert(ExpertOp op, const ExpertArgs &a, int bf16, hipStream_t s, int *workgroups)
{
    return bf16 ? run<bf16_t>(op, a, s, workgroups) : run<float>(op, a, s, workgroups);
}

}  // namespace kfac
