// Rows of 16- or 32-bit values by eights, and their form in 8 bits: E4M3 codes under one power of two per group of 128.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace cs {

typedef uint8_t u8;
typedef uint16_t u16;

constexpr int GROUP = 128;              // columns (and, in blocks, rows) that share a scale
constexpr int GROUP_LANES = GROUP / 8;  // threads of a group, eight columns each

// An access of eight neighbouring values goes by 16 bytes, by 8, or value by value (V_EACH).
enum { V_EACH = 0, V_8 = 8, V_16 = 16 };

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Eight values as they lie in memory.
template <class T>
struct alignas(16) Eight {
    T v[8];
    __device__ __forceinline__ float operator[](int i) const { return to_f32(v[i]); }
};

// Columns c .. c+7 of a row of `cols`; zero past the end.
template <class T>
__device__ __forceinline__ Eight<T> load8(const T *row, long long c, long long cols, int vec)
{
    Eight<T> e;
    if (vec != V_EACH && c + 8 <= cols) {
        if (vec == V_16) {
            uint4 *d = reinterpret_cast<uint4 *>(&e);
            const uint4 *s = reinterpret_cast<const uint4 *>(row + c);
#pragma unroll
            for (int i = 0; i < (int)sizeof(e) / 16; ++i) d[i] = s[i];
        } else {
            uint2 *d = reinterpret_cast<uint2 *>(&e);
            const uint2 *s = reinterpret_cast<const uint2 *>(row + c);
#pragma unroll
            for (int i = 0; i < (int)sizeof(e) / 8; ++i) d[i] = s[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = c + i < cols ? row[c + i] : from_f32<T>(0.0f);
    }
    return e;
}

template <class T>
__device__ __forceinline__ void store8(T *row, long long c, long long cols, int vec, const Eight<T> &e)
{
    if (vec != V_EACH && c + 8 <= cols) {
        if (vec == V_16) {
            const uint4 *s = reinterpret_cast<const uint4 *>(&e);
            uint4 *d = reinterpret_cast<uint4 *>(row + c);
#pragma unroll
            for (int i = 0; i < (int)sizeof(e) / 16; ++i) d[i] = s[i];
        } else {
            const uint2 *s = reinterpret_cast<const uint2 *>(&e);
            uint2 *d = reinterpret_cast<uint2 *>(row + c);
#pragma unroll
            for (int i = 0; i < (int)sizeof(e) / 8; ++i) d[i] = s[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) row[c + i] = e.v[i];
    }
}

// The scale of a group by the pattern of its largest magnitude, 1.m * 2^e: the quotient is at most 448 = 1.75 * 2^8.
__device__ __forceinline__ u32 scale_of(u32 most)
{
    const u32 e = most >> 23, up = (most & 0x7FFFFFu) > 0x600000u ? 1u : 0u;
    return e > 8 ? e - 8 + up : 1u;
}
__device__ __forceinline__ float scale_value(u32 s) { return __uint_as_float(s << 23); }            // 2^(s-127)
__device__ __forceinline__ float scale_inverse(u32 s) { return __uint_as_float((254u - s) << 23); } // 2^(127-s); s is at most 247

// Pattern of the largest magnitude of eight values; with `finite`, of those that are.
__device__ __forceinline__ u32 most_of(const float (&v)[8], bool finite)
{
    u32 m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const u32 b = __float_as_uint(v[i]) & 0x7FFFFFFFu;
        m = max(m, finite && b >= 0x7F800000u ? 0u : b);
    }
    return m;
}
// Largest of a group's 16 lanes. Every lane of the group is here.
__device__ __forceinline__ u32 group_most(u32 m, u32 lanes)
{
#pragma unroll
    for (int d = GROUP_LANES / 2; d > 0; d >>= 1) m = max(m, __shfl_xor_sync(lanes, m, d));
    return m;
}

// Codes of eight values under 2^(127-s). (The conversion saturates infinities, so `odd` ones are taken out of its way.)
__device__ __forceinline__ uint2 codes_of(const float (&v)[8], float inverse, bool odd)
{
    u16 q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x = v[2 * i] * inverse, y = v[2 * i + 1] * inverse;
        if (odd) {
            if (!(fabsf(v[2 * i]) <= 3.402823466e38f)) x = __uint_as_float(0x7FFFFFFFu);
            if (!(fabsf(v[2 * i + 1]) <= 3.402823466e38f)) y = __uint_as_float(0x7FFFFFFFu);
        }
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(q[i]) : "f"(y), "f"(x));
    }
    return make_uint2((u32)q[0] | (u32)q[1] << 16, (u32)q[2] | (u32)q[3] << 16);
}

__device__ __forceinline__ void store_codes(u8 *row, long long c, long long cols, uint2 q)
{
    if (c + 8 <= cols) {
        *reinterpret_cast<uint2 *>(row + c) = q;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) row[c + i] = (u8)((i < 4 ? q.x : q.y) >> (8 * (i & 3)));
    }
}

// Columns c .. c+7 of a row (zero past its end), whose group the 16 lanes around this one hold, into codes and scale. All
// lanes of the warp call it.
__device__ __forceinline__ void encode8(const float (&v)[8], u8 *codes, u8 *scales, long long c, long long cols)
{
    u32 most = group_most(most_of(v, false), 0xFFFFFFFFu);
    const bool odd = most >= 0x7F800000u;               // (the same for the group)
    if (odd) most = group_most(most_of(v, true), 0xFFFFu << (threadIdx.x & 16));
    const u32 s = scale_of(most);
    if (c < cols) {
        store_codes(codes, c, cols, codes_of(v, scale_inverse(s), odd));
        if (threadIdx.x % GROUP_LANES == 0) scales[c / GROUP] = (u8)s;
    }
}

}  // namespace cs
