// Rows of 16- or 32-bit values by eights, and their form in 8 bits: E4M3 codes under one power of two per group of 128.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "common.cuh"
#include "pieces.h"

namespace cs {

typedef uint8_t u8;
typedef uint16_t u16;

constexpr int GROUP = 128;              // columns (and, in blocks, rows) that share a scale
constexpr int GROUP_LANES = GROUP / 8;  // threads of a group, eight columns each

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
// Eight values as fp32, and eight fp32 values rounded, two at a time.
template <class T>
__device__ __forceinline__ void widen(const Eight<T> &e, float (&v)[8])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = e[i];
    } else {
        const u32 *w = reinterpret_cast<const u32 *>(&e);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            } else {
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(w + i));
                v[2 * i] = f.x;
                v[2 * i + 1] = f.y;
            }
        }
    }
}
__device__ __forceinline__ u32 pack2(float lo, float hi, __half) { const __half2 h = __floats2half2_rn(lo, hi); return *reinterpret_cast<const u32 *>(&h); }
__device__ __forceinline__ u32 pack2(float lo, float hi, __nv_bfloat16) { const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi); return *reinterpret_cast<const u32 *>(&h); }
template <class T>
__device__ __forceinline__ Eight<T> rounded(const float (&v)[8])
{
    Eight<T> e;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = v[i];
    } else {
        u32 *w = reinterpret_cast<u32 *>(&e);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack2(v[2 * i], v[2 * i + 1], T());
    }
    return e;
}

// Keeps the values as they are in registers: what has been made of them ahead of this is made anew behind it, not kept too.
template <class T>
__device__ __forceinline__ void hold(Eight<T> &e)
{
    u32 *w = reinterpret_cast<u32 *>(&e);
#pragma unroll
    for (int i = 0; i < (int)sizeof(e) / 4; ++i) asm volatile("" : "+r"(w[i]));
}
template <class T> struct Access;       // an access of four values
template <> struct Access<float> { typedef uint4 Four; };
template <> struct Access<__half> { typedef uint2 Four; };
template <> struct Access<__nv_bfloat16> { typedef uint2 Four; };

// Moves words so that they begin `by` values further on. `by` is the same for all threads of a row, so nothing here diverges.
__device__ __forceinline__ void shift_words(u32 (&w)[8], int by)           // 16-bit values: by 0 .. 7
{
    if (by & 4) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (by & 2) {
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    if (by & 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
}
__device__ __forceinline__ void shift_words(u32 (&w)[12], int by)          // 32-bit values: by 0 .. 3
{
    if (by & 2) {
#pragma unroll
        for (int i = 0; i < 10; ++i) w[i] = w[i + 2];
    }
    if (by & 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = w[i + 1];
    }
}

// Columns c .. c+7 of a row of `cols`; zero past the end. A says what the rows allow: 8 or 4 values at a time (alignment, and a
// number of columns that is a multiple of it), or one. It is fixed when compiling: a choice at every access made three to
// four times as many instructions, and kept the loads of a thread from leaving together (128 x 128 blocks of bf16: 87 us).
// Rows that begin anywhere (A = 1) are read by the aligned 16 bytes that hold the values, where those lie within the row, and
// shifted (value by value the norm of 8000 x 2047 in bf16 took 79 us, now 39; 25 for 8000 x 2048).
template <int A, class T>
__device__ __forceinline__ Eight<T> load8(const T *row, int c, int cols)
{
    Eight<T> e;
    if constexpr (A == 8) {
        uint4 *d = reinterpret_cast<uint4 *>(&e);
        const uint4 *s = reinterpret_cast<const uint4 *>(row + c);
#pragma unroll
        for (int i = 0; i < (int)sizeof(e) / 16; ++i) d[i] = c < cols ? s[i] : make_uint4(0, 0, 0, 0);
    } else if constexpr (A == 4) {
        typedef typename Access<T>::Four Four;
        Four *d = reinterpret_cast<Four *>(&e);
        const Four *s = reinterpret_cast<const Four *>(row + c);
#pragma unroll
        for (int i = 0; i < 2; ++i) d[i] = c + 4 * i < cols ? s[i] : Four{};
    } else {
        constexpr int V = 16 / (int)sizeof(T), N = (int)sizeof(e) / 16 + 1;        // values of 16 bytes; such pieces that hold the eight
        const int by = (int)(reinterpret_cast<uintptr_t>(row + c) % 16 / sizeof(T)), c0 = c - by;
        if (c0 >= 0 && c0 + (by ? N : N - 1) * V <= cols) {
            alignas(16) u32 w[4 * N];
            const uint4 *s = reinterpret_cast<const uint4 *>(row + c0);
#pragma unroll
            for (int i = 0; i < N; ++i) *reinterpret_cast<uint4 *>(w + 4 * i) = i < N - 1 || by ? s[i] : make_uint4(0, 0, 0, 0);
            shift_words(w, by);
            u32 *d = reinterpret_cast<u32 *>(&e);
#pragma unroll
            for (int i = 0; i < (int)sizeof(e) / 4; ++i) d[i] = w[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) e.v[i] = c + i < cols ? row[c + i] : from_f32<T>(0.0f);
        }
    }
    return e;
}

// The same in two steps, so that several loads can be under way: ask8() loads, take8() makes the eight values of it. Of rows that begin
// anywhere the aligned pieces are loaded that hold the values. What else lies in such 16 bytes is read with them, of the neighbouring rows or
// between them, but no piece without a value of the row, and nothing out of the matrix (`off`: where the row begins in it, `total`: where it
// ends). 32-bit values, which would take three pieces, come as eights at once.
template <class T>
struct Pieces {
    static constexpr int V = PIECE, N = 2;              // values of a piece, pieces
    uint4 p[N];
};
template <int A, class T> using Asked = typename std::conditional<A == 1 && sizeof(T) == 2, Pieces<T>, Eight<T>>::type;

template <int A, class T>
__device__ __forceinline__ Asked<A, T> ask8(const T *base, long long off, long long total, int c, int cols)
{
    if constexpr (A != 1 || sizeof(T) == 4) {
        return load8<A>(base + off, c, cols);
    } else {
        typedef Pieces<T> P;
        P a;
        const long long at = off + c;
        const int by = (int)(reinterpret_cast<uintptr_t>(base + at) % 16 / sizeof(T)), n = second_piece(by, c, cols) ? P::N : P::N - 1;
        const long long start = at - by;
#pragma unroll
        for (int i = 0; i < P::N; ++i) a.p[i] = make_uint4(0, 0, 0, 0);
        if (c < cols) {
            if (start >= 0 && start + n * P::V <= total) {
                const uint4 *s = reinterpret_cast<const uint4 *>(base + start);
#pragma unroll
                for (int i = 0; i < P::N; ++i)
                    if (i < n) a.p[i] = s[i];
            } else {                    // the first and the last pieces of the matrix
                T *v = reinterpret_cast<T *>(a.p);
#pragma unroll
                for (int i = 0; i < P::N * P::V; ++i)
                    if (start + i >= 0 && start + i < total && i < n * P::V) v[i] = base[start + i];
            }
        }
        return a;
    }
}
template <int A, class T>
__device__ __forceinline__ Eight<T> take8(const Asked<A, T> &a, const T *base, long long off, int c, int cols)
{
    if constexpr (A != 1 || sizeof(T) == 4) {
        return a;
    } else {
        typedef Pieces<T> P;
        u32 w[4 * P::N];
#pragma unroll
        for (int i = 0; i < P::N; ++i) {
            w[4 * i] = a.p[i].x;
            w[4 * i + 1] = a.p[i].y;
            w[4 * i + 2] = a.p[i].z;
            w[4 * i + 3] = a.p[i].w;
        }
        shift_words(w, (int)(reinterpret_cast<uintptr_t>(base + off + c) % 16 / sizeof(T)));
        Eight<T> e;
        u32 *d = reinterpret_cast<u32 *>(&e);
#pragma unroll
        for (int i = 0; i < (int)sizeof(e) / 4; ++i) d[i] = w[i];
        if (c + 8 > cols) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i >= cols) e.v[i] = from_f32<T>(0.0f);
        }
        return e;
    }
}

// The other way; of rows that begin anywhere whole warps write (store8_warp).
template <int A, class T>
__device__ __forceinline__ void store8(T *row, int c, int cols, const Eight<T> &e)
{
    static_assert(A == 8 || A == 4, "access width");
    if constexpr (A == 8) {
        const uint4 *s = reinterpret_cast<const uint4 *>(&e);
        uint4 *d = reinterpret_cast<uint4 *>(row + c);
        if (c < cols) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(e) / 16; ++i) d[i] = s[i];
        }
    } else {
        typedef typename Access<T>::Four Four;
        const Four *s = reinterpret_cast<const Four *>(&e);
        Four *d = reinterpret_cast<Four *>(row + c);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (c + 4 * i < cols) d[i] = s[i];
    }
}

// The same by a whole warp whose lanes hold eights that follow one another in a row. Where rows begin anywhere, the values go through
// the warp's `turn` (32 eights) and out 32 neighbours at a time, not with 16 bytes between the lanes of an access.
template <int A, class T>
__device__ __forceinline__ void store8_warp(T *row, int c, int cols, const Eight<T> &e, Eight<T> *turn)
{
    if constexpr (A != 1) {
        store8<A>(row, c, cols, e);
    } else {
        const int lane = threadIdx.x & 31, first = c - lane * 8;
        __syncwarp();
        turn[lane] = e;
        __syncwarp();
        const T *s = reinterpret_cast<const T *>(turn);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (first + i * 32 + lane < cols) row[first + i * 32 + lane] = s[i * 32 + lane];
    }
}
// Room for the turns of a CTA's warps.
template <int A, class T, int BLOCK> struct Turns {
    static constexpr int N = A == 1 ? BLOCK : 1;
};

// The scale of a group by its largest magnitude 1.m * 2^e: the quotient is at most 448 = 1.75 * 2^8.
__device__ __forceinline__ u32 scale_of(float most)
{
    const u32 b = __float_as_uint(most), s = (b + 0x1FFFFFu) >> 23;     // (e, or e + 1 for m > 0x600000)
    return s > 9 ? s - 8 : 1u;
}
__device__ __forceinline__ float scale_value(u32 s) { return __uint_as_float(s << 23); }            // 2^(s-127)
__device__ __forceinline__ float scale_inverse(u32 s) { return __uint_as_float((254u - s) << 23); } // 2^(127-s); s is at most 247

// Largest magnitude; no number if one of them is none.
__device__ __forceinline__ float most3(float a, float b, float c)
{
    float m;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}
__device__ __forceinline__ float most2(float a, float b)
{
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
__device__ __forceinline__ float most_of(const float (&v)[8]) { return most3(most3(most3(v[0], v[1], v[2]), v[3], v[4]), most3(v[5], v[6], v[7]), 0.0f); }
// ... of those that are finite
__device__ __forceinline__ float most_finite(const float (&v)[8])
{
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fabsf(v[i]) <= 3.402823466e38f ? fmaxf(m, fabsf(v[i])) : m;
    return m;
}
// Largest of a group's 16 lanes. Every lane of `lanes` is here.
__device__ __forceinline__ float group_most(float m, u32 lanes)
{
#pragma unroll
    for (int d = GROUP_LANES / 2; d > 0; d >>= 1) m = most2(m, __shfl_xor_sync(lanes, m, d));
    return m;
}
__device__ __forceinline__ bool is_odd(float most) { return !(most <= 3.402823466e38f); }

// Codes of eight values under 2^(127-s).
__device__ __forceinline__ uint2 codes_of(const float (&v)[8], float inverse)
{
    u16 q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(q[i]) : "f"(v[2 * i + 1] * inverse), "f"(v[2 * i] * inverse));
    return make_uint2((u32)q[0] | (u32)q[1] << 16, (u32)q[2] | (u32)q[3] << 16);
}
// (The conversion saturates infinities: they are made NaN ahead of it.)
__device__ __forceinline__ void odd_to_nan(float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (!(fabsf(v[i]) <= 3.402823466e38f)) v[i] = __uint_as_float(0x7FFFFFFFu);
}

// Rows of codes are 16-byte aligned whatever their width.
template <int A>
__device__ __forceinline__ void store_codes(u8 *row, int c, int cols, uint2 q)
{
    if (A == 8 || c + 8 <= cols) {
        *reinterpret_cast<uint2 *>(row + c) = q;
    } else if (A == 4) {
        *reinterpret_cast<u32 *>(row + c) = q.x;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) row[c + i] = (u8)((i < 4 ? q.x : q.y) >> (8 * (i & 3)));
    }
}

// Columns c .. c+7 of a row (zero past its end), whose group the 16 lanes around this one hold, into codes and scale. All
// lanes of the warp call it.
template <int A>
__device__ __forceinline__ void encode8(float (&v)[8], u8 *codes, u8 *scales, int c, int cols)
{
    float most = group_most(most_of(v), 0xFFFFFFFFu);
    if (is_odd(most)) {                                 // (the same for the group)
        most = group_most(most_finite(v), 0xFFFFu << (threadIdx.x & 16));
        odd_to_nan(v);
    }
    const u32 s = scale_of(most);
    if (c < cols) {
        store_codes<A>(codes, c, cols, codes_of(v, scale_inverse(s)));
        if (threadIdx.x % GROUP_LANES == 0) scales[(u32)c / GROUP] = (u8)s;
    }
}

}  // namespace cs
