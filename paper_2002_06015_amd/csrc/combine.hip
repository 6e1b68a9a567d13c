// The join of the results of a token's experts, out = residual + sum_j gate_j y_j, and its gradients dy_j = gate_j dout,
// dgate_j = <dout, y_j>.
//
// Sums in fp32 in the order of j, one rounding; the products of a gate's gradient are added up by one wave or one workgroup, in an
// order that depends on the sizes only (which of the two: run_grad).  Both are bound by memory: every element is read or written once.  32768 tokens of two
// choices, 2048 channels, bf16: 94 - 100 us forward (5.4 - 5.7 TB/s), 109 - 116 with both gradients (5.8 - 6.2); 2051 x 4 x 1001 in fp32,
// no row aligned: 9 and 15 us.
#include <algorithm>

#include "elements.h"
#include "token_internal.h"

namespace kfac {

namespace {

// 2^log threads a token (workgroups of 256: several tokens, or a token in several steps), eight elements a thread, FAN choices' rows in flight
// (EXACT: a token has as many).
template <typename T, typename S, int FAN, bool EXACT, bool SHORT>
__global__ __launch_bounds__(256) void combine_kernel(const CombineArgs a, int log)
{
    const long long stripe = (long long)gridDim.x << (8 - log);
    for (long long token = ((long long)blockIdx.x << (8 - log)) + (threadIdx.x >> log); token < a.tokens; token += stripe)
      for (int c = 8 * (int)(threadIdx.x & ((1 << log) - 1)); c < a.dim; c += 8 << log) {
        const int there = a.dim - c;
        float sum[8], v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) sum[q] = 0.f;
        const T *y = (const T *)a.y + token * a.fan * a.ldy;
        const float *gate = a.gate + token * a.fan;
        Raw8<S> res;
        if (a.r) res.template load<SHORT>((const S *)a.r + token * a.ldr, c, a.dim);
        for (int j0 = 0; j0 < (EXACT ? FAN : a.fan); j0 += FAN) {
            Raw8<T> raw[FAN];
            float g[FAN];
#pragma unroll
            for (int j = 0; j < FAN; ++j)
                if (EXACT || j0 + j < a.fan) {
                    raw[j].template load<SHORT>(y + (j0 + j) * a.ldy, c, a.dim);
                    g[j] = a.gate ? gate[j0 + j] : 1.f;
                }
#pragma unroll
            for (int j = 0; j < FAN; ++j)
                if (EXACT || j0 + j < a.fan) {
                    raw[j].get(v);
#pragma unroll
                    for (int q = 0; q < 8; ++q) sum[q] = fmaf(g[j], v[q], sum[q]);
                }
        }
        if (a.r) {
            res.get(v);
#pragma unroll
            for (int q = 0; q < 8; ++q) sum[q] += v[q];
        }
        store8((S *)a.out + token * a.ldo + c, there, sum);
    }
}

// THREADS threads for FAN choices of a token, whose rows are in flight together (four of them: 2051 x 4 x 1001 fp32 18 us instead of 15).
template <typename T, typename S, int THREADS, int FAN, bool SHORT>
__global__ __launch_bounds__(256) void combine_grad_kernel(const CombineArgs a)
{
    __shared__ float parts[4 * FAN];
    const int me = threadIdx.x % THREADS, lane = threadIdx.x & 63;
    const int sets = (a.fan + FAN - 1) / FAN;   // of choices, a token
    const long long all = (long long)a.tokens * sets, stripe = (long long)gridDim.x * (256 / THREADS);
    for (long long set = (long long)blockIdx.x * (256 / THREADS) + threadIdx.x / THREADS; set < all; set += stripe) {
        const long long token = sets == 1 ? set : set / sets;
        const int j0 = sets == 1 ? 0 : FAN * (int)(set - token * sets);
        const S *dout = (const S *)a.dout + token * a.ldd;
        const long long choice = token * a.fan + j0;
        float g[FAN], dot[FAN];
#pragma unroll
        for (int j = 0; j < FAN; ++j) {
            g[j] = a.gate && a.dy && j0 + j < a.fan ? a.gate[choice + j] : 1.f;
            dot[j] = 0.f;
        }
        for (int c = 8 * me; c < a.dim; c += 8 * THREADS) {
            float d[8], v[8];
            Raw8<S> raw_d;
            Raw8<T> raw_y[FAN];
            raw_d.template load<SHORT>(dout, c, a.dim);
            if (a.dgate)
#pragma unroll
                for (int j = 0; j < FAN; ++j)
                    if (j0 + j < a.fan) raw_y[j].template load<SHORT>((const T *)a.y + (choice + j) * a.ldy, c, a.dim);
            raw_d.get(d);
#pragma unroll
            for (int j = 0; j < FAN; ++j) {
                if (j0 + j >= a.fan) break;
                if (a.dgate) {
                    raw_y[j].get(v);
#pragma unroll
                    for (int q = 0; q < 8; ++q) dot[j] = fmaf(d[q], v[q], dot[j]);
                }
                if (a.dy) {
#pragma unroll
                    for (int q = 0; q < 8; ++q) v[q] = g[j] * d[q];
                    store8((T *)a.dy + (choice + j) * a.lddy + c, a.dim - c, v);
                }
            }
        }
        if (!a.dgate) continue;
#pragma unroll
        for (int j = 0; j < FAN; ++j)
            for (int o = 32; o > 0; o >>= 1) dot[j] += __shfl_xor(dot[j], o);
        if constexpr (THREADS == 64) {
#pragma unroll
            for (int j = 0; j < FAN; ++j)
                if (lane == j && j0 + j < a.fan) a.dgate[choice + j] = dot[j];
        } else {
            __syncthreads();
            if (lane == 0)
#pragma unroll
                for (int j = 0; j < FAN; ++j) parts[(threadIdx.x >> 6) * FAN + j] = dot[j];
            __syncthreads();
            if (threadIdx.x < FAN && j0 + (int)threadIdx.x < a.fan)
                a.dgate[choice + threadIdx.x] = parts[threadIdx.x] + parts[FAN + threadIdx.x] + parts[2 * FAN + threadIdx.x] + parts[3 * FAN + threadIdx.x];
        }
    }
}

template <typename T, typename S>
hipError_t run(const CombineArgs &a, hipStream_t s)
{
    int log = 0;
    while (log < 8 && (8 << log) < a.dim) ++log;
    const long long wgs = ((long long)a.tokens + (256 >> log) - 1) >> (8 - log);
    const dim3 grid((unsigned)std::min(wgs, 1LL << 20));   // a launch takes less than 2^32 threads
    if (a.dim < 8) combine_kernel<T, S, 1, false, true><<<grid, dim3(256), 0, s>>>(a, log);
    else if (a.fan == 1) combine_kernel<T, S, 1, true, false><<<grid, dim3(256), 0, s>>>(a, log);
    else if (a.fan == 2) combine_kernel<T, S, 2, true, false><<<grid, dim3(256), 0, s>>>(a, log);
    else combine_kernel<T, S, 4, false, false><<<grid, dim3(256), 0, s>>>(a, log);
    return hipGetLastError();
}

template <typename T, typename S, int THREADS, bool SHORT>
hipError_t run_grad(const CombineArgs &a, hipStream_t s)
{
    constexpr int per = 256 / THREADS;
    const long long sets = (long long)a.tokens * ((a.fan + 1) / 2);
    const dim3 grid((unsigned)std::min((sets + per - 1) / per, 1LL << 20)), block(256);   // a launch takes less than 2^32 threads
    if (a.fan <= 1) combine_grad_kernel<T, S, THREADS, 1, SHORT><<<grid, block, 0, s>>>(a);
    else combine_grad_kernel<T, S, THREADS, 2, SHORT><<<grid, block, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, typename S>
hipError_t run_grad(const CombineArgs &a, hipStream_t s)
{
    if (a.dim < 8) return run_grad<T, S, 64, true>(a, s);
    // A wave for a pair of choices where it has two steps at most and there are enough (2051 x 4 x 1001 fp32: 15 us, 19 with a workgroup; 20000 x 1
    // x 512: 14 and 20), otherwise a workgroup (32768 x 2 x 2048 bf16: 116 us, 122 with a wave; 1024 x 2 x 4096: 8 and 11).
    const long long sets = (long long)a.tokens * ((a.fan + 1) / 2);
    return a.dim <= 512 || (a.dim <= 1024 && sets >= 4096) ? run_grad<T, S, 64, false>(a, s) : run_grad<T, S, 256, false>(a, s);
}

}  // namespace

hipError_t launch_combine(const CombineArgs &a, int bf16, int out_bf16, hipStream_t s)
{
    if (bf16) return out_bf16 ? run<bf16_bits, bf16_bits>(a, s) : run<bf16_bits, float>(a, s);
    return out_bf16 ? run<float, bf16_bits>(a, s) : run<float, float>(a, s);
}

hipError_t launch_combine_grad(const CombineArgs &a, int bf16, int out_bf16, hipStream_t s)
{
    if (bf16) return out_bf16 ? run_grad<bf16_bits, bf16_bits>(a, s) : run_grad<bf16_bits, float>(a, s);
    return out_bf16 ? run_grad<float, bf16_bits>(a, s) : run_grad<float, float>(a, s);
}

}  // namespace kfac
