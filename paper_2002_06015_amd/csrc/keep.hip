// Activations in 8 bits: blocks of 32 adjacent elements of a row under a power-of-two scale, e4m3 values.
//
// 2^e is the least power with max |x| <= 448 2^e over the block's finite elements, so nothing is cut off and an element above
// 2^-6 of that range is held to four bits (half a step: 2^-4 of it).  Scaling by a power of two is exact: the one rounding is the
// conversion, and what is held, q 2^e with e >= -117, is exact in bf16 and fp32.  Both directions are bound by memory: 16384 x 2048
// bf16, inputs that no cache holds: 21 us (4.9 TB/s), 25 with eight elements a thread; back 18 us, 5.6 TB/s (values of a repeated call: 17 and 17).
#include <algorithm>

#include "elements.h"
#include "token_internal.h"

namespace kfac {

namespace {

// 2^log threads a row (workgroups of 256: several rows, or a row in several steps), sixteen elements a thread; two adjacent threads: a block.
// Threads behind a row's end or the last row do their part, so that the lanes of a block are all there, and store nothing.
template <typename T, bool SHORT>
__global__ __launch_bounds__(256) void keep_kernel(const KeepArgs a, int log)
{
    const long long stripe = (long long)gridDim.x << (8 - log);
    for (long long r0 = (long long)blockIdx.x << (8 - log); r0 < a.rows; r0 += stripe) {
        const long long mine = r0 + (threadIdx.x >> log), row = mine < a.rows ? mine : a.rows - 1;
        for (int c0 = 0; c0 < a.cols; c0 += 16 << log) {
            const int c = c0 + 16 * (int)(threadIdx.x & ((1 << log) - 1)), there = mine < a.rows ? a.cols - c : 0;
            float v[2][8];
            Raw8<T> raw[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) raw[h].template load<SHORT>((const T *)a.x + row * a.ldx, c + 8 * h, a.cols);
#pragma unroll
            for (int h = 0; h < 2; ++h) raw[h].get(v[h]);
            uint2_u q[2];
            const int byte = to_8_bits(v, q);
            if (there > 0) store_bytes(a.q + row * a.ldq + c, there, q);
            if (there > 0 && (threadIdx.x & 1) == 0) a.scales[row * a.lds + c / 32] = (unsigned char)byte;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void restore_kernel(const KeepArgs a, int log)
{
    const long long stripe = (long long)gridDim.x << (8 - log);
    for (long long row = ((long long)blockIdx.x << (8 - log)) + (threadIdx.x >> log); row < a.rows; row += stripe) {
        long long from = row;
        if (a.gather) {
            const int choice = a.order ? a.order[row] : (int)row;
            from = (unsigned)min(max(choice, 0), (int)a.rows - 1) / (unsigned)a.fan;
        }
        for (int c = 16 * (int)(threadIdx.x & ((1 << log) - 1)); c < a.cols; c += 16 << log) {
            uint2_u q[2];
            load_bytes(a.q + from * a.ldq + c, a.cols - c, q);
            const int byte = a.scales[from * a.lds + c / 32];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[8];
                from_8_bits(q[h], byte, v);
                store8((T *)a.back + row * a.ldx + c + 8 * h, a.cols - c - 8 * h, v);
            }
        }
    }
}

template <typename K>
hipError_t run(K kernel, const KeepArgs &a, hipStream_t s)
{
    int log = 1;
    while (log < 8 && (16 << log) < a.cols) ++log;
    const long long wgs = (a.rows + (256 >> log) - 1) >> (8 - log);
    kernel<<<dim3((unsigned)std::min(wgs, 1LL << 20)), dim3(256), 0, s>>>(a, log);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_keep(const KeepArgs &a, int bf16, hipStream_t s)
{
    if (a.cols < 8) return bf16 ? run(keep_kernel<bf16_bits, true>, a, s) : run(keep_kernel<float, true>, a, s);
    return bf16 ? run(keep_kernel<bf16_bits, false>, a, s) : run(keep_kernel<float, false>, a, s);
}
hipError_t launch_restore(const KeepArgs &a, int bf16, hipStream_t s)
{
    return bf16 ? run(restore_kernel<bf16_bits>, a, s) : run(restore_kernel<float>, a, s);
}

}  // namespace kfac
