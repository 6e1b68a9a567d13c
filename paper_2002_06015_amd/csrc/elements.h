// Eight adjacent elements of a row, in memory as fp32, bf16 or e4m3, in registers as fp32.  Any alignment to whole elements.
#pragma once

#include <hip/hip_runtime.h>

namespace kfac {

typedef float float4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short ushort8_u __attribute__((ext_vector_type(8), aligned(2)));
typedef unsigned uint2_u __attribute__((ext_vector_type(2), aligned(1)));
typedef unsigned uint4_u __attribute__((ext_vector_type(4), aligned(1)));
typedef unsigned short bf16_bits;

template <typename T> struct Element;
template <> struct Element<float> {
    static __device__ __forceinline__ float get(const float *p) { return *p; }
    static __device__ __forceinline__ void put(float *p, float v) { *p = v; }
    static __device__ __forceinline__ float round(float v) { return v; }
};
template <> struct Element<bf16_bits> {
    static __device__ __forceinline__ float get(const bf16_bits *p) { return __uint_as_float((unsigned)*p << 16); }
    static __device__ __forceinline__ void put(bf16_bits *p, float v) { *p = __builtin_bit_cast(bf16_bits, (__bf16)v); }
    static __device__ __forceinline__ float round(float v) { return (float)(__bf16)v; }
};

// Eight elements of a row from place c on, zeros behind its end.  load() has no branches and only sends the loads out: where the row ends
// inside the eight, or before them, its last eight are loaded, and get() moves them.  (A branch around a load, or a conversion next to it, makes
// every load wait for the one before it.)  SHORT: rows of less than eight elements, one by one.
template <typename T>
struct Raw8 {
    float4_u a, b;   // bf16: the 16 bytes are in a
    int back;
    template <bool SHORT>
    __device__ __forceinline__ void load(const T *row, int c, int cols)
    {
        if constexpr (SHORT) {
            back = 0;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? Element<T>::get(row + c + j) : 0.f;
            if constexpr (sizeof(T) == 2) {
                ushort8_u r;
#pragma unroll
                for (int j = 0; j < 8; ++j) r[j] = (bf16_bits)(__float_as_uint(v[j]) >> 16);
                a = __builtin_bit_cast(float4_u, r);
            } else {
                a = float4_u{v[0], v[1], v[2], v[3]};
                b = float4_u{v[4], v[5], v[6], v[7]};
            }
        } else {
            const int from = min(c, cols - 8);
            back = min(c - from, 8);
            if constexpr (sizeof(T) == 2) {
                a = __builtin_bit_cast(float4_u, *(const ushort8_u *)(row + from));
            } else {
                a = *(const float4_u *)(row + from);
                b = *(const float4_u *)(row + from + 4);
            }
        }
    }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        if constexpr (sizeof(T) == 2) {
            const ushort8_u r = __builtin_bit_cast(ushort8_u, a);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __uint_as_float((unsigned)r[j] << 16);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) { v[j] = a[j]; v[4 + j] = b[j]; }
        }
        if (back)
#pragma unroll
            for (int s = 8; s > 0; s >>= 1)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = back & s ? (j + s < 8 ? v[j + s] : 0.f) : v[j];
    }
};

template <typename T>
__device__ __forceinline__ void load8(const T *__restrict__ p, float (&v)[8])
{
    Raw8<T> r;
    r.template load<false>(p, 0, 8);
    r.get(v);
}

template <typename T>
__device__ __forceinline__ void store8(T *__restrict__ p, int there, const float (&v)[8])
{
    if (there >= 8) {
        if constexpr (sizeof(T) == 2) {
            ushort8_u r;
#pragma unroll
            for (int j = 0; j < 8; ++j) r[j] = __builtin_bit_cast(bf16_bits, (__bf16)v[j]);
            *(ushort8_u *)p = r;
        } else {
            float4_u a, b;
#pragma unroll
            for (int j = 0; j < 4; ++j) { a[j] = v[j]; b[j] = v[4 + j]; }
            *(float4_u *)p = a;
            *(float4_u *)(p + 4) = b;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < there) Element<T>::put(p + j, v[j]);
    }
}

// ---- blocks of 32 in 8 bits: lanes 4 i .. 4 i + 3 of a wave hold a block, eight elements each ------------
// What a block's scale goes by: the bits of its largest finite magnitude.
__device__ __forceinline__ unsigned finite_bits(float v)
{
    const unsigned a = __float_as_uint(v) & 0x7FFFFFFFu;
    return a < 0x7F800000u ? a : 0u;
}
template <int CTRL>
__device__ __forceinline__ unsigned from_lane(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true); }

// e + 127 for the least e in [-117, 119] with magnitude <= 448 2^e (448 = 1.75 2^8)
__device__ __forceinline__ int scale_byte(unsigned magnitude)
{
    const int e = (int)(magnitude >> 23) - 8 + ((magnitude & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return min(max(e, 127 - 117), 127 + 119);
}
__device__ __forceinline__ float power_of_two(int byte) { return __uint_as_float((unsigned)byte << 23); }

// Eight elements over a scale.
__device__ __forceinline__ void in_8_bits(const float (&v)[8], int byte, uint2_u &q)
{
    const float inverse = power_of_two(254 - byte);
    float u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float w = v[j] * inverse;
        u[j] = (__float_as_uint(v[j]) & 0x7F800000u) == 0x7F800000u ? __uint_as_float(0x7FC00000u) : __builtin_amdgcn_fmed3f(w, -448.f, 448.f);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        int r = __builtin_amdgcn_cvt_pk_fp8_f32(u[4 * j], u[4 * j + 1], 0, false);
        q[j] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(u[4 * j + 2], u[4 * j + 3], r, true);
    }
}

// All lanes of a wave call these.  v: zeros behind the row's end.  They return the block's scale byte; q: the bytes.
__device__ __forceinline__ int to_8_bits(const float (&v)[8], uint2_u &q)
{
    unsigned high = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) high = max(high, finite_bits(v[j]));
    high = max(high, from_lane<0xB1>(high));   // quad_perm 1 0 3 2
    high = max(high, from_lane<0x4E>(high));   // quad_perm 2 3 0 1
    const int byte = scale_byte(high);
    in_8_bits(v, byte, q);
    return byte;
}

// Sixteen elements a lane: lanes 2 i and 2 i + 1 hold a block.
__device__ __forceinline__ int to_8_bits(const float (&v)[2][8], uint2_u (&q)[2])
{
    unsigned high = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 8; ++j) high = max(high, finite_bits(v[h][j]));
    high = max(high, from_lane<0xB1>(high));   // quad_perm 1 0 3 2
    const int byte = scale_byte(high);
    in_8_bits(v[0], byte, q[0]);
    in_8_bits(v[1], byte, q[1]);
    return byte;
}

// The values of eight bytes under a scale.
__device__ __forceinline__ void from_8_bits(const uint2_u &q, int byte, float (&v)[8])
{
    const float scale = power_of_two(byte);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[j], true);
        v[4 * j] = lo[0] * scale;
        v[4 * j + 1] = lo[1] * scale;
        v[4 * j + 2] = hi[0] * scale;
        v[4 * j + 3] = hi[1] * scale;
    }
}

// The first `there` of eight bytes.
__device__ __forceinline__ void store_bytes(unsigned char *p, int there, const uint2_u &q)
{
    if (there >= 8) {
        *(uint2_u *)p = q;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < there) p[j] = (unsigned char)(q[j >> 2] >> (8 * (j & 3)));
    }
}
__device__ __forceinline__ uint2_u load_bytes(const unsigned char *p, int there)
{
    if (there >= 8) return *(const uint2_u *)p;
    uint2_u q = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < there) q[j >> 2] |= (unsigned)p[j] << (8 * (j & 3));
    return q;
}

// The same of sixteen.
__device__ __forceinline__ void store_bytes(unsigned char *p, int there, const uint2_u (&q)[2])
{
    if (there >= 16) {
        *(uint4_u *)p = uint4_u{q[0][0], q[0][1], q[1][0], q[1][1]};
    } else {
        store_bytes(p, there, q[0]);
        store_bytes(p + 8, there - 8, q[1]);
    }
}
__device__ __forceinline__ void load_bytes(const unsigned char *p, int there, uint2_u (&q)[2])
{
    if (there >= 16) {
        const uint4_u r = *(const uint4_u *)p;
        q[0] = uint2_u{r[0], r[1]};
        q[1] = uint2_u{r[2], r[3]};
    } else {
        q[0] = load_bytes(p, there);
        q[1] = load_bytes(p + 8, there - 8);
    }
}

}  // namespace kfac
