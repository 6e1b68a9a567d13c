// Dropout from a counter: y = r + keep * x / (1 - p), the same call without r for the gradient.
//
// The mask is a function of (seed, offset, index of the element in the [rows, cols] matrix) and is never stored:
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC 2011) gives 128 bits for
// the counter (index / 8, offset) under the key `seed`; an element takes 16 of them and is kept where they are not below
// round(65536 p).  (16 bits: one block of the generator serves 16 bytes of bf16, and p is met to 2^-17; the scale is that of
// the rounded p, so the mean is exact.)  Arithmetic in fp32, one rounding at the end.  Memory bound:
// 65537 x 1000 fp32 with a residual 130 us (6.0 TB/s), 8192 x 2048 bf16 16 us with and 13 without one; the twenty 32 x 32 -> 64 bit
// products of a block run beside its loads.
#include "token_internal.h"

namespace kfac {

namespace {

typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short u16x8_u __attribute__((ext_vector_type(8), aligned(2)));

__device__ __forceinline__ uint4 philox(unsigned long long block, unsigned long long offset, unsigned long long seed)
{
    unsigned c0 = (unsigned)block, c1 = (unsigned)(block >> 32), c2 = (unsigned)offset, c3 = (unsigned)(offset >> 32);
    unsigned k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (unsigned)(b >> 32) ^ c1 ^ k0;
        c1 = (unsigned)b;
        c2 = (unsigned)(a >> 32) ^ c3 ^ k1;
        c3 = (unsigned)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

template <typename T>
__device__ __forceinline__ void load8(const T *__restrict__ p, float (&v)[8])
{
    if constexpr (sizeof(T) == 2) {
        const u16x8_u r = *(const u16x8_u *)p;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float((unsigned)r[j] << 16);
    } else {
        const f32x4_u a = *(const f32x4_u *)p, b = *(const f32x4_u *)(p + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) { v[j] = a[j]; v[4 + j] = b[j]; }
    }
}

template <typename T>
__device__ __forceinline__ void store8(T *__restrict__ p, const float (&v)[8])
{
    if constexpr (sizeof(T) == 2) {
        u16x8_u r;
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = __builtin_bit_cast(unsigned short, (__bf16)v[j]);
        *(u16x8_u *)p = r;
    } else {
        f32x4_u a, b;
#pragma unroll
        for (int j = 0; j < 4; ++j) { a[j] = v[j]; b[j] = v[4 + j]; }
        *(f32x4_u *)p = a;
        *(f32x4_u *)(p + 4) = b;
    }
}

// A thread: the elements of one row that share a block of the generator, eight unless the row starts or ends inside it.
// Rows that follow each other without a gap are one row.
template <typename T, bool RES>
__global__ __launch_bounds__(256) void dropout_kernel(const DropoutArgs a, unsigned per_row, unsigned long long units)
{
    for (unsigned long long u = (unsigned long long)blockIdx.x * 256 + threadIdx.x; u < units; u += (unsigned long long)gridDim.x * 256) {
        const unsigned long long row = a.rows == 1 ? 0 : u / per_row;
        const unsigned long long begin = row * a.cols, end = begin + a.cols;         // indices of the row's elements
        const unsigned long long block = (begin >> 3) + (u - row * per_row);
        const long long c0 = (long long)(block * 8) - (long long)begin;              // column of the block's first element
        if (block * 8 >= end) continue;
        const uint4 w = philox(block, a.offset, a.seed);
        const unsigned word[4] = {w.x, w.y, w.z, w.w};
        const T *x = (const T *)a.x + row * a.ldx, *r = (const T *)a.r + row * a.ldr;
        T *y = (T *)a.y + row * a.ldy;
        float v[8], q[8];
        const bool whole = c0 >= 0 && c0 + 8 <= a.cols;
        if (whole) {
            load8(x + c0, v);
            if constexpr (RES) load8(r + c0, q);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = q[j] = 0.f;
                if (c0 + j >= 0 && c0 + j < a.cols) {
                    if constexpr (sizeof(T) == 2) {
                        v[j] = __uint_as_float((unsigned)x[c0 + j] << 16);
                        if constexpr (RES) q[j] = __uint_as_float((unsigned)r[c0 + j] << 16);
                    } else {
                        v[j] = x[c0 + j];
                        if constexpr (RES) q[j] = r[c0 + j];
                    }
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned bits = j & 1 ? word[j >> 1] >> 16 : word[j >> 1] & 0xFFFFu;
            const float kept = bits >= a.threshold ? v[j] * a.factor : 0.f;          // (a dropped infinity or NaN is a zero)
            v[j] = RES ? q[j] + kept : kept;
        }
        if (whole) {
            store8(y + c0, v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + j >= 0 && c0 + j < a.cols) {
                    if constexpr (sizeof(T) == 2) y[c0 + j] = __builtin_bit_cast(unsigned short, (__bf16)v[j]);
                    else y[c0 + j] = v[j];
                }
        }
    }
}

template <typename T>
hipError_t run(DropoutArgs a, hipStream_t s)
{
    if (a.ldx == a.cols && a.ldy == a.cols && (!a.r || a.ldr == a.cols)) {
        a.cols *= a.rows;
        a.rows = 1;
    }
    // blocks of the generator that a row can touch
    const unsigned long long per_row = a.rows == 1 || a.cols % 8 == 0 ? (a.cols + 7) / 8 : (a.cols + 7) / 8 + 1;
    const unsigned long long units = per_row * a.rows, wgs = (units + 255) / 256;
    const dim3 grid((unsigned)(wgs < (1 << 20) ? wgs : (1 << 20)));   // a launch takes less than 2^32 threads; the kernel goes on from there
    if (a.r) dropout_kernel<T, true><<<grid, dim3(256), 0, s>>>(a, (unsigned)per_row, units);
    else dropout_kernel<T, false><<<grid, dim3(256), 0, s>>>(a, (unsigned)per_row, units);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs &a, int bf16, hipStream_t s)
{
    return bf16 ? run<unsigned short>(a, s) : run<float>(a, s);
}

}  // namespace kfac
