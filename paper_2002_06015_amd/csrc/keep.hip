// Activations in 8 bits: blocks of 32 adjacent elements of a row under a power-of-two scale, e4m3 values.
//
// 2^e is the least power with max |x| <= 448 2^e over the block's finite elements, so nothing is cut off and an element above
// 2^-6 of that range is held to four bits (half a step: 2^-4 of it).  Scaling by a power of two is exact: the one rounding is the
// conversion, and what is held, q 2^e with e >= -117, is exact in bf16 and fp32.  Both directions are bound by memory.
#include "elements.h"
#include "token_internal.h"

namespace kfac {

namespace {

// A thread: eight elements of a row; four adjacent threads: a block.  Threads behind the last one do their part with zeros, so that the
// lanes of a block are all there.
template <typename T>
__global__ __launch_bounds__(256) void keep_kernel(const KeepArgs a, unsigned per_row, unsigned long long units)
{
    for (unsigned long long first = (unsigned long long)blockIdx.x * 256; first < units; first += (unsigned long long)gridDim.x * 256) {
        const unsigned long long u = first + threadIdx.x, row = u / per_row;
        const int c = 8 * (int)(u - row * per_row), there = u < units ? a.cols - c : 0;
        float v[8];
        load8((const T *)a.x + row * a.ldx + c, there, v);
        uint2_u q;
        const int byte = to_8_bits(v, q);
        if (there > 0) store_bytes(a.q + row * a.ldq + c, there, q);
        if (there > 0 && (threadIdx.x & 3) == 0) a.scales[row * a.lds + c / 32] = (unsigned char)byte;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void restore_kernel(const KeepArgs a, unsigned per_row, unsigned long long units)
{
    for (unsigned long long u = (unsigned long long)blockIdx.x * 256 + threadIdx.x; u < units; u += (unsigned long long)gridDim.x * 256) {
        const unsigned long long row = u / per_row;
        const int c = 8 * (int)(u - row * per_row), there = a.cols - c;
        if (there <= 0) continue;   // (a row has whole blocks of threads)
        long long from = (long long)row;
        if (a.gather) {
            const int choice = a.order ? a.order[row] : (int)row;
            from = (unsigned)min(max(choice, 0), (int)a.rows - 1) / (unsigned)a.fan;
        }
        float v[8];
        from_8_bits(load_bytes(a.q + from * a.ldq + c, there), a.scales[from * a.lds + c / 32], v);
        store8((T *)a.back + row * a.ldx + c, there, v);
    }
}

template <typename K>
hipError_t run(K kernel, const KeepArgs &a, hipStream_t s)
{
    const unsigned per_row = 4u * (unsigned)((a.cols + 31) / 32);
    const unsigned long long units = (unsigned long long)a.rows * per_row, wgs = (units + 255) / 256;
    kernel<<<dim3((unsigned)(wgs < (1 << 20) ? wgs : (1 << 20))), dim3(256), 0, s>>>(a, per_row, units);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_keep(const KeepArgs &a, int bf16, hipStream_t s) { return bf16 ? run(keep_kernel<bf16_bits>, a, s) : run(keep_kernel<float>, a, s); }
hipError_t launch_restore(const KeepArgs &a, int bf16, hipStream_t s)
{
    return bf16 ? run(restore_kernel<bf16_bits>, a, s) : run(restore_kernel<float>, a, s);
}

}  // namespace kfac
