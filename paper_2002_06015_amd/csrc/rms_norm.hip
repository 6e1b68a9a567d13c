// Root-mean-square norm of a residual stream, and its gradients.
//
//   h = x + residual,  r = 1 / sqrt(mean h^2 + eps),  u = r h,  y = gamma u
//   dh = dstream + r (g - u mean(g u)),  g = gamma dy;   dgamma = sum over tokens of dy u;   F = mean over tokens of (dy u)^2
// h is rounded to the type of the stream before the norm is taken of it, so that the gradient, which reads the written h, belongs to
// exactly what was computed; everything else is fp32, rounded once.  A row is read once and stays in the registers of the
// wave (or workgroup) that has it.  Columns are summed over a workgroup's rows in its registers, then over the workgroups in the order
// of their numbers by a second launch.  Bound by memory.
#include <algorithm>

#include "elements.h"
#include "token_internal.h"

namespace kfac {

namespace {

// The sum over the THREADS threads of a row, in all of them.
// parts: LDS, N THREADS / 64 of the row's own
template <int THREADS, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float *parts)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) v[i] += __shfl_xor(v[i], o);
    if constexpr (THREADS > 64) {
        constexpr int W = THREADS / 64;
        __syncthreads();   // what was there has been read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) parts[i * W + (threadIdx.x % THREADS >> 6)] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) v[i] += parts[i * W + w];
        }
    }
}

__device__ __forceinline__ float inverse_root(float squares, int dim, float eps) { return 1.f / sqrtf(squares / (float)dim + eps); }

// THREADS threads a row, CH chunks of eight elements each; workgroups of at least 256 threads.
template <typename T, typename S, int THREADS, int CH, bool SHORT>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void norm_kernel(const NormArgs a)
{
    constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
    __shared__ float parts[ROWS][THREADS / 64];
    const int me = threadIdx.x % THREADS;
    for (long long first = (long long)blockIdx.x * ROWS; first < a.n; first += (long long)gridDim.x * ROWS) {
        const long long mine = first + threadIdx.x / THREADS, row = mine < a.n ? mine : a.n - 1;   // (all threads meet at the barriers)
        const int dim = mine < a.n ? a.dim : 0;   // what is stored
        float h[CH][8], sum[1] = {0.f};
        Raw8<T> raw_x[CH];
        Raw8<S> raw_r[CH];
        Raw8<float> raw_g[CH];
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = 8 * (me + THREADS * k);
            raw_x[k].template load<SHORT>((const T *)a.x + row * a.ldx, c, a.dim);
            if (a.r) raw_r[k].template load<SHORT>((const S *)a.r + row * a.ldr, c, a.dim);
            raw_g[k].template load<SHORT>(a.gamma, c, a.dim);
        }
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            raw_x[k].get(h[k]);
            if (a.r) {
                float r[8];
                raw_r[k].get(r);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[k][j] = Element<S>::round(h[k][j] + r[j]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[0] = fmaf(h[k][j], h[k][j], sum[0]);
        }
        row_sums<THREADS>(sum, parts[threadIdx.x / THREADS]);
        const float r = inverse_root(sum[0], a.dim, a.eps);
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = 8 * (me + THREADS * k), there = dim - c;
            if (a.h) store8((S *)a.h + row * a.ldh + c, there, h[k]);
            float g[8];
            raw_g[k].get(g);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] *= h[k][j] * r;
            if (a.y) store8((T *)a.y + row * a.ldy + c, there, g);
            if (a.q) {
                uint2_u q;
                const int byte = to_8_bits(g, q);
                if (there > 0) store_bytes(a.q + row * a.ldq + c, there, q);
                if (there > 0 && (threadIdx.x & 3) == 0) a.scales[row * a.lds + c / 32] = (unsigned char)byte;
            }
        }
    }
}

// COLUMNS: sums of the columns too, one row of them for each workgroup (in the order in which it has its rows, four at least: norm_parts).
// 16384 rows 2048, bf16 and fp32 stream, with both: 99 us, 4.7 TB/s, with 512 workgroups; 136 with 256, 112 with 384, 106 with 768,
// 111 with 1024 (and more to add up).  2053 rows 1001 in fp32: 12 us, in four rows for each sum as in two or one.
template <typename T, typename S, int THREADS, int CH, bool COLUMNS, bool SHORT>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void norm_grad_kernel(const NormGradArgs a)
{
    constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
    __shared__ float parts[ROWS][2 * (THREADS / 64)], columns[COLUMNS && ROWS > 1 ? 8 * 256 : 1];
    const int me = threadIdx.x % THREADS, stripe = gridDim.x * ROWS;
    float first[COLUMNS ? CH : 1][8], second[COLUMNS ? CH : 1][8];
    if constexpr (COLUMNS)
#pragma unroll
        for (int k = 0; k < CH; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) first[k][j] = second[k][j] = 0.f;
    // a row is on its way while the one before it is worked on
    Raw8<S> raw_h[CH], raw_r[CH];
    Raw8<T> raw_d[CH];
    auto fetch = [&](long long next) {
        const long long row = next < a.n ? next : a.n - 1;   // (all threads meet at the barriers)
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = 8 * (me + THREADS * k);
            raw_h[k].template load<SHORT>((const S *)a.h + row * a.ldh, c, a.dim);
            raw_d[k].template load<SHORT>((const T *)a.dy + row * a.lddy, c, a.dim);
            if (a.r && a.dh) raw_r[k].template load<SHORT>((const S *)a.r + row * a.ldr, c, a.dim);
        }
    };
    float gamma[CH][8];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = 8 * (me + THREADS * k);
        Raw8<float> raw;
        raw.template load<SHORT>(a.gamma, c, a.dim);
        raw.get(gamma[k]);
    }
    const int mine = threadIdx.x / THREADS;
    fetch((long long)blockIdx.x * ROWS + mine);
    for (long long row0 = (long long)blockIdx.x * ROWS; row0 < a.n; row0 += stripe) {
        const long long row = row0 + mine;
        const int dim = row < a.n ? a.dim : 0;
        float h[CH][8], d[CH][8], o[CH][8], sums[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            raw_h[k].get(h[k]);
            raw_d[k].get(d[k]);
            if (a.r && a.dh) raw_r[k].get(o[k]);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j) o[k][j] = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sums[0] = fmaf(h[k][j], h[k][j], sums[0]);
                sums[1] = fmaf(gamma[k][j] * d[k][j], h[k][j], sums[1]);
            }
        }
        fetch(row + stripe);
        row_sums<THREADS>(sums, parts[mine]);
        const float r = inverse_root(sums[0], a.dim, a.eps), along = r * r * (sums[1] / (float)a.dim);
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = 8 * (me + THREADS * k);
            if (COLUMNS && dim > 0)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float p = d[k][j] * (h[k][j] * r);
                    first[k][j] += p;
                    second[k][j] = fmaf(p, p, second[k][j]);
                }
            if (a.dh && dim > c) {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[k][j] = fmaf(r, gamma[k][j] * d[k][j] - h[k][j] * along, o[k][j]);
                store8((S *)a.dh + row * a.lddh + c, dim - c, o[k]);
            }
        }
    }
    if constexpr (COLUMNS) {
        float *const out = a.partial + 2LL * blockIdx.x * a.dim;
#pragma unroll
        for (int k = 0; k < CH; ++k)
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                const int c = 8 * (me + THREADS * k);
                float *const v = which ? second[k] : first[k];
                if constexpr (ROWS > 1) {   // element j of thread t at 256 j + t
                    __syncthreads();
#pragma unroll
                    for (int j = 0; j < 8; ++j) columns[256 * j + threadIdx.x] = v[j];
                    __syncthreads();
                    if ((int)threadIdx.x >= THREADS) continue;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int w = 1; w < ROWS; ++w) v[j] += columns[256 * j + THREADS * w + threadIdx.x];
                }
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < a.dim) out[(long long)which * a.dim + c + j] = v[j];
            }
    }
}

// 32 columns a workgroup, 32 threads a column: the parts one after the other, eight of them on their way together (512 parts of 2048 columns 4.8 us,
// 7.0 with one), then the threads.
__global__ __launch_bounds__(1024) void norm_join_kernel(const NormGradArgs a, int parts)
{
    __shared__ float sums[2][32][33];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float v[2] = {0.f, 0.f};
    if (c < a.dim)
        for (int p0 = group; p0 < parts; p0 += 32 * 8) {
            float one[8], two[8];   // in flight together
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const long long p = min(p0 + 32 * i, parts - 1);
                one[i] = a.partial[2 * p * a.dim + c];
                two[i] = a.partial[(2 * p + 1) * a.dim + c];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (p0 + 32 * i < parts) {
                    v[0] += one[i];
                    v[1] += two[i];
                }
        }
    sums[0][group][lane] = v[0];
    sums[1][group][lane] = v[1];
    __syncthreads();
    if (group < 2 && c < a.dim) {
        float total = 0.f;
#pragma unroll
        for (int q = 0; q < 32; ++q) total += sums[group][q][lane];
        if (group == 0) {
            if (a.dgamma) a.dgamma[c] = total;
        } else if (a.F && a.n > 0) {
            const float mean = total / (float)a.n;
            a.F[c] = a.decay == 0.f ? mean : fmaf(1.f - a.decay, mean, a.decay * a.F[c]);
        }
    }
}

// A launch takes less than 2^32 threads; the kernels go on from there.
unsigned workgroups(int n, int rows) { return (unsigned)std::min((n + rows - 1) / rows, 1 << 20); }

template <typename T, typename S, int THREADS, int CH, bool SHORT = false>
hipError_t run(const NormArgs &a, hipStream_t s)
{
    constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
    norm_kernel<T, S, THREADS, CH, SHORT><<<dim3(workgroups(a.n, ROWS)), dim3(THREADS < 256 ? 256 : THREADS), 0, s>>>(a);
    return hipGetLastError();
}
template <typename T, typename S>
hipError_t run(const NormArgs &a, hipStream_t s)
{
    // one chunk a thread up to 8192 (16384 rows 2048, bf16 and fp32 stream, 8 bits beside: 73 us, 90 with a wave a row and four chunks a thread)
    if (a.dim < 8) return run<T, S, 64, 1, true>(a, s);
    if (a.dim <= 512) return run<T, S, 64, 1>(a, s);
    if (a.dim <= 1024) return run<T, S, 128, 1>(a, s);
    if (a.dim <= 2048) return run<T, S, 256, 1>(a, s);
    if (a.dim <= 4096) return run<T, S, 512, 1>(a, s);
    if (a.dim <= 8192) return run<T, S, 1024, 1>(a, s);
    return run<T, S, 1024, 2>(a, s);
}

int rows_at_once(int dim) { return dim <= 512 ? 4 : dim <= 1024 ? 2 : 1; }

template <typename T, typename S, int THREADS, int CH, bool SHORT = false>
hipError_t run_grad(const NormGradArgs &a, hipStream_t s)
{
    constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
    const dim3 block(THREADS < 256 ? 256 : THREADS);
    if (a.dgamma || a.F) norm_grad_kernel<T, S, THREADS, CH, true, SHORT><<<dim3((unsigned)norm_parts(a.n, a.dim)), block, 0, s>>>(a);
    else norm_grad_kernel<T, S, THREADS, CH, false, SHORT><<<dim3(workgroups(a.n, ROWS)), block, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T, typename S>
hipError_t run_grad(const NormGradArgs &a, hipStream_t s)
{
    if (a.dim < 8) return run_grad<T, S, 64, 1, true>(a, s);
    if (a.dim <= 512) return run_grad<T, S, 64, 1>(a, s);
    if (a.dim <= 1024) return run_grad<T, S, 128, 1>(a, s);
    if (a.dim <= 2048) return run_grad<T, S, 256, 1>(a, s);
    if (a.dim <= 4096) return run_grad<T, S, 512, 1>(a, s);
    if (a.dim <= 8192) return run_grad<T, S, 1024, 1>(a, s);
    return run_grad<T, S, 1024, 2>(a, s);
}

}  // namespace

int norm_parts(int n, int dim)
{
    const int rows = rows_at_once(dim), most = (n + 4 * rows - 1) / (4 * rows);   // four rows at least for a row of sums
    return most < 1 ? 1 : most > 512 ? 512 : most;
}

hipError_t launch_norm(const NormArgs &a, int bf16, int stream_bf16, hipStream_t s)
{
    if (bf16) return stream_bf16 ? run<bf16_bits, bf16_bits>(a, s) : run<bf16_bits, float>(a, s);
    return stream_bf16 ? run<float, bf16_bits>(a, s) : run<float, float>(a, s);
}

hipError_t launch_norm_grad(const NormGradArgs &a, int bf16, int stream_bf16, hipStream_t s)
{
    if (bf16) return stream_bf16 ? run_grad<bf16_bits, bf16_bits>(a, s) : run_grad<bf16_bits, float>(a, s);
    return stream_bf16 ? run_grad<float, bf16_bits>(a, s) : run_grad<float, float>(a, s);
}

hipError_t launch_norm_join(const NormGradArgs &a, hipStream_t s)
{
    norm_join_kernel<<<dim3((unsigned)((a.dim + 31) / 32)), dim3(1024), 0, s>>>(a, a.n > 0 ? norm_parts(a.n, a.dim) : 0);
    return hipGetLastError();
}

}  // namespace kfac
