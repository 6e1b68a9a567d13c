// Embedding lookup with scaling, and the gradient of its table by sorted tokens.
//
// Lookup: out[i] = scale * T[ids[i]].  A thread takes a piece of a row, eight elements where both are bf16 and four otherwise; the
// pieces of all rows follow each other.  Reads the distinct rows, writes all.
//
// Gradient: dT[v] = scale * sum over the positions of token v, added in fp32 in the order of the positions, without atomics.
// The positions come sorted by token.  A wave takes a run of `chunk` sorted positions and one 64-lane piece of the columns,
// keeps the running sum in registers and writes a row where the token changes.  A token whose positions cross runs leaves its
// part of the sum in scratch, and the join adds the parts in order.  Rows of tokens that do not occur are zeros, which the sort's
// launches write beside the sort.  Memory bound: the gradients are read once, the table's gradient is written once, rows of tokens
// that occur twice.  131071 x 1024 bf16, 65536 tokens: lookup 90 us (4.4 TB/s), gradient 77 (sort and zeros) + 90 (sums, 5 TB/s) + 18
// (join); 8191 x 1024, 32000 tokens: lookup 9, gradient 22 + 11 + 9, where the zeros (131 MB) are the floor.
#include "token_internal.h"

namespace kfac {

namespace {

typedef unsigned short bf16_t;
typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));                     // 16 bytes at an element's alignment
typedef unsigned short u16x8_u __attribute__((ext_vector_type(8), aligned(2)));
typedef unsigned short u16x4_u __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float from_bf16(bf16_t v) { return __uint_as_float((unsigned)v << 16); }
// to nearest, ties to even; NaN stays NaN
__device__ __forceinline__ bf16_t to_bf16(float v) { return __builtin_bit_cast(bf16_t, (__bf16)v); }

// W adjacent elements as floats (W = 8: bf16, 4: float), the first `c` of them; ONCE: nobody reads them again
template <typename T, int W, bool ONCE = false>
__device__ __forceinline__ void load_piece(const T *__restrict__ p, int c, float (&v)[W])
{
    if (c >= W) {
        if constexpr (sizeof(T) == 2 && W == 8) {
            const u16x8_u r = ONCE ? __builtin_nontemporal_load((const u16x8_u *)p) : *(const u16x8_u *)p;
#pragma unroll
            for (int j = 0; j < W; ++j) v[j] = from_bf16(r[j]);
        } else if constexpr (sizeof(T) == 2) {
            const u16x4_u r = *(const u16x4_u *)p;
#pragma unroll
            for (int j = 0; j < W; ++j) v[j] = from_bf16(r[j]);
        } else {
#pragma unroll
            for (int q = 0; q < W / 4; ++q) {
                const f32x4_u *at = (const f32x4_u *)((const float *)p + 4 * q);
                const f32x4_u r = ONCE ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[4 * q + j] = r[j];
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < W; ++j) {
            v[j] = 0.f;
            if (j < c) {
                if constexpr (sizeof(T) == 2) v[j] = from_bf16(p[j]);
                else v[j] = p[j];
            }
        }
    }
}

template <typename T, int W>
__device__ __forceinline__ void store_piece(T *__restrict__ p, int c, const float (&v)[W])
{
    if (c >= W) {
        if constexpr (sizeof(T) == 2 && W == 8) {
            u16x8_u r;
#pragma unroll
            for (int j = 0; j < W; ++j) r[j] = to_bf16(v[j]);
            *(u16x8_u *)p = r;
        } else if constexpr (sizeof(T) == 2) {
            u16x4_u r;
#pragma unroll
            for (int j = 0; j < W; ++j) r[j] = to_bf16(v[j]);
            *(u16x4_u *)p = r;
        } else {
#pragma unroll
            for (int q = 0; q < W / 4; ++q) {
                f32x4_u r;
#pragma unroll
                for (int j = 0; j < 4; ++j) r[j] = v[4 * q + j];
                *(f32x4_u *)((float *)p + 4 * q) = r;
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < W; ++j)
            if (j < c) {
                if constexpr (sizeof(T) == 2) p[j] = to_bf16(v[j]);
                else p[j] = v[j];
            }
    }
}

// A thread: W adjacent columns of one row.
template <typename ID, typename TT, typename TO>
__global__ __launch_bounds__(256) void embedding_kernel(const ID *__restrict__ ids, long long pieces, int per_row, int vocab, int dim,
                                                        const TT *__restrict__ table, long long ldt, float scale, TO *__restrict__ out,
                                                        long long ldo)
{
    constexpr int W = sizeof(TT) == 2 && sizeof(TO) == 2 ? 8 : 4;
    for (long long u = (long long)blockIdx.x * 256 + threadIdx.x; u < pieces; u += (long long)gridDim.x * 256) {
        const long long row = u / per_row;
        const int c0 = W * (int)(u - row * per_row);
        const ID id = ids[row];
        float v[W];
        if (id >= 0 && id < (ID)vocab) load_piece<TT, W>(table + (long long)id * ldt + c0, dim - c0, v);
        else
#pragma unroll
            for (int j = 0; j < W; ++j) v[j] = 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] *= (id >= 0 && id < (ID)vocab) ? scale : 0.f;
        store_piece<TO, W>(out + row * ldo + c0, dim - c0, v);
    }
}

template <int W>
__device__ __forceinline__ void write_row(const EmbeddingGrad &a, int key, int count, int c0, const float (&sum)[W])
{
    float *row = a.dW + (long long)key * a.dim + c0;
    float v[W];
    if (a.accumulate) load_piece<float, W>(row, a.dim - c0, v);
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = a.accumulate ? fmaf(a.scale, sum[j], v[j]) : a.scale * sum[j];
    store_piece<float, W>(row, a.dim - c0, v);
    if (c0 == 0 && a.A) a.A[key] = fmaf(a.share, (float)count, a.A[key]);
}

// A wave: a run of sorted positions, 64 W columns.
template <typename T, bool ONCE>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const EmbeddingGrad a, int col_tiles, int chunks)
{
    constexpr int W = sizeof(T) == 2 ? 8 : 4, AHEAD = 8;
    const int lane = threadIdx.x & 63;
    const long long unit = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = (int)(unit / col_tiles), c0 = ((int)(unit - (long long)c * col_tiles) * 64 + lane) * W;
    if (c >= chunks) return;
    const int i0 = c * a.chunk, cnt = min(a.chunk, a.n - i0);
    // keys and positions of the run, one a lane; neighbours on either side
    const int mine = min(i0 + min(lane, cnt - 1), a.n - 1);
    const int my_key = a.keys[mine], my_pos = a.pos[mine];
    const int before = i0 > 0 ? a.keys[i0 - 1] : -1, after = i0 + cnt < a.n ? a.keys[i0 + cnt] : -1;
    const T *g = (const T *)a.g;
    float sum[W];
#pragma unroll
    for (int j = 0; j < W; ++j) sum[j] = 0.f;
    int start = 0, key = __builtin_amdgcn_readlane(my_key, 0);
    if (key >= a.vocab) return;
    auto flush = [&](int end) {   // positions [start, end) of this run have `key`
        if (c0 < a.dim) {
            const bool from = start > 0 || before != key, to = end < cnt || after != key;
            if (from && to) {
                write_row<W>(a, key, end - start, c0, sum);
            } else {   // the part that goes on from the run before, or the one that goes on behind this run
                store_piece<float, W>(a.partial + ((long long)2 * c + (from ? 1 : 0)) * a.dim + c0, a.dim - c0, sum);
            }
        }
#pragma unroll
        for (int j = 0; j < W; ++j) sum[j] = 0.f;
        start = end;
    };
    for (int r0 = 0; r0 < cnt; r0 += AHEAD) {
        float v[AHEAD][W];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int p = __builtin_amdgcn_readlane(my_pos, min(r0 + u, cnt - 1));
            if (c0 < a.dim) load_piece<T, W, ONCE>(g + (long long)p * a.ld + c0, a.dim - c0, v[u]);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (r0 + u >= cnt) break;
            const int k = __builtin_amdgcn_readlane(my_key, r0 + u);
            if (k != key) {
                flush(r0 + u);
                key = k;
                if (key >= a.vocab) return;   // sorted: no token from here on
            }
#pragma unroll
            for (int j = 0; j < W; ++j) sum[j] += v[u][j];
        }
    }
    flush(cnt);
}

// Tokens whose positions cross runs: a wave for every run in which such a token starts and 256 columns adds its parts, in order.
// A token of more than kLongParts parts is left to the whole workgroup, which adds up a share of the parts in each wave.
constexpr int kJoinWaves = 8, kLongParts = 24;
__global__ __launch_bounds__(64 * kJoinWaves) void embedding_join_kernel(const EmbeddingGrad a, int chunks)
{
    __shared__ float part[kJoinWaves][64][4];
    __shared__ int is_long[kJoinWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c0 = (blockIdx.y * 64 + lane) * 4;
    // Parts of the token that goes on behind run c and starts in it (0: there is none), and its positions.  The lanes look at the ends of
    // 64 runs at a time: a search through all keys would be a chain of a dozen loads.
    auto look = [&](int c, int &key, int &count) {
        if (c >= chunks) return 0;
        const int first = c * a.chunk, last = min(first + a.chunk, a.n) - 1;
        key = a.keys[last];
        const int mine = a.keys[min(first + lane, last)], next = a.keys[min(last + 1, a.n - 1)], before = a.keys[max(first - 1, 0)];
        if (key >= a.vocab || last + 1 >= a.n || next != key) return 0;
        const int here = __popcll(__ballot(first + lane <= last && mine == key));
        if (here == last + 1 - first && c > 0 && before == key) return 0;                     // it came from before
        int parts = 1;   // runs that the token fills to their end
        for (;;) {
            const int end = (c + parts + lane + 1) * a.chunk - 1;
            const unsigned long long through = __ballot(end < a.n && a.keys[min(end, a.n - 1)] == key);
            if (through == ~0ULL) { parts += 64; continue; }
            parts += __ffsll(~through) - 1;
            break;
        }
        const int tail = (c + parts) * a.chunk;
        const int there = __popcll(__ballot(lane < a.chunk && tail + lane < a.n && a.keys[min(tail + lane, a.n - 1)] == key));
        count = here + (parts - 1) * a.chunk + there;
        return there > 0 ? parts + 1 : parts;
    };
    auto add = [&](int c, int p0, int p1, float (&sum)[4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = 0.f;
        if (c0 < a.dim) {
#pragma unroll 8
            for (int p = p0; p < p1; ++p) {
                float v[4];
                load_piece<float, 4>(a.partial + ((long long)2 * (c + p) + (p == 0 ? 1 : 0)) * a.dim + c0, a.dim - c0, v);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] += v[j];
            }
        }
    };
    auto write = [&](int key, int count, const float (&sum)[4]) {
        if (c0 < a.dim) write_row<4>(a, key, count, c0, sum);
    };
    int key = 0, count = 0;
    float sum[4];
    const int mine = blockIdx.x * kJoinWaves + wave, parts = look(mine, key, count);
    if (lane == 0) is_long[wave] = parts > kLongParts;
    if (parts > 0 && parts <= kLongParts) {
        add(mine, 0, parts, sum);
        write(key, count, sum);
    }
    __syncthreads();
    for (int w = 0; w < kJoinWaves; ++w) {
        if (!is_long[w]) continue;
        const int c = blockIdx.x * kJoinWaves + w, all = look(c, key, count), per = (all + kJoinWaves - 1) / kJoinWaves;
        add(c, min(wave * per, all), min(wave * per + per, all), sum);
#pragma unroll
        for (int j = 0; j < 4; ++j) part[wave][lane][j] = sum[j];
        __syncthreads();
        if (wave == 0) {
            for (int q = 1; q < kJoinWaves; ++q)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] += part[q][lane][j];
            write(key, count, sum);
        }
        __syncthreads();
    }
}

template <typename ID, typename TT, typename TO>
hipError_t lookup(const ID *ids, int n, int vocab, int dim, const void *table, long long ldt, float scale, void *out, long long ldo, hipStream_t s)
{
    constexpr int W = sizeof(TT) == 2 && sizeof(TO) == 2 ? 8 : 4;
    const int per_row = (dim + W - 1) / W;
    const long long pieces = (long long)n * per_row;
    const long long wgs = (pieces + 255) / 256;
    embedding_kernel<ID, TT, TO><<<dim3((unsigned)(wgs < (1 << 20) ? wgs : (1 << 20))), dim3(256), 0, s>>>(
        ids, pieces, per_row, vocab, dim, (const TT *)table, ldt, scale, (TO *)out, ldo);
    return hipGetLastError();
}

template <typename ID>
hipError_t lookup_types(const ID *ids, int n, int vocab, int dim, int table_bf16, const void *table, long long ldt, float scale, int out_bf16,
                        void *out, long long ldo, hipStream_t s)
{
    if (table_bf16) return out_bf16 ? lookup<ID, bf16_t, bf16_t>(ids, n, vocab, dim, table, ldt, scale, out, ldo, s)
                                    : lookup<ID, bf16_t, float>(ids, n, vocab, dim, table, ldt, scale, out, ldo, s);
    return out_bf16 ? lookup<ID, float, bf16_t>(ids, n, vocab, dim, table, ldt, scale, out, ldo, s)
                    : lookup<ID, float, float>(ids, n, vocab, dim, table, ldt, scale, out, ldo, s);
}

}  // namespace

hipError_t launch_embedding(const void *ids, int id_bits, int n, int vocab, int dim, int table_bf16, const void *table, long long ldt,
                            float scale, int out_bf16, void *out, long long ldo, hipStream_t s)
{
    return id_bits == 64 ? lookup_types((const long long *)ids, n, vocab, dim, table_bf16, table, ldt, scale, out_bf16, out, ldo, s)
                         : lookup_types((const int *)ids, n, vocab, dim, table_bf16, table, ldt, scale, out_bf16, out, ldo, s);
}

// Short runs where there are few positions, so that there are waves enough; long ones leave fewer parts to join.  The whole gradient of a
// table of 32000 tokens in bf16, runs of 8 and of 32 positions: 256 wide 36 and 47 us for 8192 positions, 59 and 62 for 32768, 75 and 68
// for 65536; 1024 wide 40 and 50, 87 and 79, 122 and 105.  (In fp32 34 and 39, 59 and 58, 75 and 62; 40 and 41, 96 and 89, 143 and 122.)
constexpr int kShortRuns = 32768;
int embedding_chunk(int n) { return n <= kShortRuns ? 8 : 32; }
int embedding_most_chunks(int n)
{
    const int here = (n + embedding_chunk(n) - 1) / embedding_chunk(n);
    return n <= kShortRuns || here > kShortRuns / 8 ? here : kShortRuns / 8;
}

hipError_t launch_embedding_sum(const EmbeddingGrad &a, hipStream_t s)
{
    const int chunks = (a.n + a.chunk - 1) / a.chunk;
    const int piece = 64 * (a.bf16 ? 8 : 4), col_tiles = (a.dim + piece - 1) / piece;
    const long long wgs = ((long long)chunks * col_tiles + 3) / 4;
    const dim3 grid((unsigned)wgs), block(256);
    // gradients that the caches cannot hold are read past them, which leaves the caches to the rows that are written (131071 x 1024 bf16:
    // 89 us, 125 through them); smaller ones may still be there from their writing (8191 x 1024: 11 us, 13 past them)
    const bool once = (long long)a.n * a.dim * (a.bf16 ? 2 : 4) > (64LL << 20);
    if (a.bf16) {
        if (once) embedding_sum_kernel<bf16_t, true><<<grid, block, 0, s>>>(a, col_tiles, chunks);
        else embedding_sum_kernel<bf16_t, false><<<grid, block, 0, s>>>(a, col_tiles, chunks);
    } else {
        if (once) embedding_sum_kernel<float, true><<<grid, block, 0, s>>>(a, col_tiles, chunks);
        else embedding_sum_kernel<float, false><<<grid, block, 0, s>>>(a, col_tiles, chunks);
    }
    return hipGetLastError();
}

hipError_t launch_embedding_join(const EmbeddingGrad &a, hipStream_t s)
{
    const int chunks = (a.n + a.chunk - 1) / a.chunk;
    embedding_join_kernel<<<dim3((chunks + kJoinWaves - 1) / kJoinWaves, (a.dim + 255) / 256), dim3(64 * kJoinWaves), 0, s>>>(a, chunks);
    return hipGetLastError();
}

}  // namespace kfac
