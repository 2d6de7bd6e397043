// AdamW over a tensor list with moments in 32 or in 8 bits, and the norm of the gradient it uses.
//
// Both are one pass over the list. A warp takes 256 elements at a time, which is also the block
// that shares a scale of the 8-bit states: lane l holds the quads at 4l and at 128 + 4l, so every
// load and store of the warp is contiguous in every type (512 bytes of fp32, 256 of a 16-bit type,
// 128 of codes), and the largest magnitude of a block is one warp reduction.
// The tensors' descriptors travel in the kernel's parameters: no copy to the device ahead of the
// launch, and nothing of a call outlives it.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "common.cuh"

namespace cs {

typedef unsigned short u16;

constexpr int LIST_CHUNK = 256;          // elements of a warp's step and of a block of 8-bit states
constexpr int NORM_GRID_MAX = 640;       // CTAs of the norm
constexpr int LIST_SMALL = 40, LIST_LARGE = 360;     // tensors whose descriptors fit 4 KB resp. 32 KB of parameters

enum { GT_F32 = 0, GT_F16 = 1, GT_BF16 = 2 };        // CONDENSA_DTYPE_*
enum { ST_32 = 0, ST_8_NEAREST = 1, ST_8_STOCHASTIC = 2 };   // moments, and how those in 8 bits are rounded

struct ListDesc {
    float *w;
    const float *theta;
    const float *lam;
    const void *grad;
    void *m;
    void *v;
    float *m_scale;
    float *v_scale;
    u16 *w_h;
    long long numel;
    u32 item0;        // first work item of the tensor
    u32 vec_ok;       // every array allows the quad accesses
};

struct ListScalars {
    float mu, grad_scale;
    float beta1, beta2, c1, c2, decay, step_size, root_corr, eps;
    const float *clip;      // norm, coefficient, finite
    int T;
    u32 n_items;
    int chunks;             // chunks of LIST_CHUNK elements per warp in a work item
    int copy_type;          // of w_h
    int t0;                 // the launch's first tensor in the list
    u64 key;                // of the call's random bits (stochastic rounding of the 8-bit states)
};

template <int CAP>
struct ListParams {
    ListScalars s;
    ListDesc d[CAP];
};
static_assert(sizeof(ListParams<LIST_SMALL>) <= 4096 && sizeof(ListParams<LIST_LARGE>) <= 32764, "kernel parameters");

template <class P>
__device__ __forceinline__ int list_owner(const P &p, u32 item)
{
    int lo = 0, hi = p.s.T - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.d[mid].item0 <= item) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// CTAs of k_adamw that an SM holds: four where 64 registers hold a step without spilling.
__host__ __device__ constexpr int adamw_ctas(int states, bool penalty)
{
    return states == ST_32 || (states == ST_8_STOCHASTIC && penalty) ? 3 : 4;
}

// Eight values of a warp's chunk that this lane holds: elements 4l..4l+3 and 128+4l..128+4l+3,
// `left` elements from the chunk's start on exist.
struct Oct { float x[8]; };

__device__ __forceinline__ Oct load_f32(const float *p, int lane, long long left, bool vec)
{
    Oct o;
    if (vec) {
        const float4 a = reinterpret_cast<const float4 *>(p)[lane], b = reinterpret_cast<const float4 *>(p)[32 + lane];
        o = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = (i >> 2) * 128 + 4 * lane + (i & 3);
            o.x[i] = e < left ? p[e] : 0.0f;
        }
    }
    return o;
}

__device__ __forceinline__ void store_f32(float *p, const Oct &o, int lane, long long left, bool vec)
{
    if (vec) {
        reinterpret_cast<float4 *>(p)[lane] = make_float4(o.x[0], o.x[1], o.x[2], o.x[3]);
        reinterpret_cast<float4 *>(p)[32 + lane] = make_float4(o.x[4], o.x[5], o.x[6], o.x[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = (i >> 2) * 128 + 4 * lane + (i & 3);
            if (e < left) p[e] = o.x[i];
        }
    }
}

template <int GT>
__device__ __forceinline__ float widen(u16 b)
{
    return GT == GT_F16 ? __half2float(__ushort_as_half(b)) : __uint_as_float((u32)b << 16);
}

template <int GT>
__device__ __forceinline__ Oct load_grad(const void *base, long long e0, int lane, long long left, bool vec)
{
    if (GT == GT_F32) return load_f32((const float *)base + e0, lane, left, vec);
    const u16 *p = (const u16 *)base + e0;
    Oct o;
    if (vec) {
        const uint2 a = reinterpret_cast<const uint2 *>(p)[lane], b = reinterpret_cast<const uint2 *>(p)[32 + lane];
        const u32 q[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o.x[2 * i] = widen<GT>((u16)(q[i] & 0xFFFF));
            o.x[2 * i + 1] = widen<GT>((u16)(q[i] >> 16));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = (i >> 2) * 128 + 4 * lane + (i & 3);
            o.x[i] = e < left ? widen<GT>(p[e]) : 0.0f;
        }
    }
    return o;
}

// A lane's eight gradients of a whole chunk as they lie in memory.
template <int GT>
struct Raw {
    uint4 v[GT == GT_F32 ? 2 : 1];
    __device__ __forceinline__ void load(const char *p, int lane)
    {
        if (GT == GT_F32) {
            v[0] = __ldg(reinterpret_cast<const uint4 *>(p) + lane);
            v[GT == GT_F32 ? 1 : 0] = __ldg(reinterpret_cast<const uint4 *>(p) + 32 + lane);
        } else {
            const uint2 a = __ldg(reinterpret_cast<const uint2 *>(p) + lane), b = __ldg(reinterpret_cast<const uint2 *>(p) + 32 + lane);
            v[0] = make_uint4(a.x, a.y, b.x, b.y);
        }
    }
    __device__ __forceinline__ Oct widened() const
    {
        Oct o;
        const u32 q[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
        if (GT == GT_F32) {
            const uint4 b = v[GT == GT_F32 ? 1 : 0];
            const u32 r[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o.x[i] = __uint_as_float(q[i]);
                o.x[4 + i] = __uint_as_float(r[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o.x[2 * i] = widen<GT>((u16)(q[i] & 0xFFFF));
                o.x[2 * i + 1] = widen<GT>((u16)(q[i] >> 16));
            }
        }
        return o;
    }
};

__device__ __forceinline__ u32 pack_copy(float a, float b, int type)
{
    if (type == GT_F16) {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const u32 *>(&h);
    }
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const u32 *>(&h);
}

__device__ __forceinline__ void store_copy(u16 *p, const Oct &o, int type, int lane, long long left, bool vec)
{
    u32 q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = pack_copy(o.x[2 * i], o.x[2 * i + 1], type);
    if (vec) {
        reinterpret_cast<uint2 *>(p)[lane] = make_uint2(q[0], q[1]);
        reinterpret_cast<uint2 *>(p)[32 + lane] = make_uint2(q[2], q[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = (i >> 2) * 128 + 4 * lane + (i & 3);
            if (e < left) p[e] = (u16)(q[i >> 1] >> (16 * (i & 1)));
        }
    }
}

// ------------------------------------------------------------------ 8-bit states
__device__ __forceinline__ void load_codes(const uint8_t *p, u32 (&c)[2], int lane, long long left, bool vec)
{
    if (vec) {
        c[0] = reinterpret_cast<const u32 *>(p)[lane];
        c[1] = reinterpret_cast<const u32 *>(p)[32 + lane];
    } else {
        c[0] = c[1] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = (i >> 2) * 128 + 4 * lane + (i & 3);
            if (e < left) c[i >> 2] |= (u32)p[e] << (8 * (i & 3));
        }
    }
}

__device__ __forceinline__ void store_codes(uint8_t *p, const u32 (&c)[2], int lane, long long left, bool vec)
{
    if (vec) {
        reinterpret_cast<u32 *>(p)[lane] = c[0];
        reinterpret_cast<u32 *>(p)[32 + lane] = c[1];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = (i >> 2) * 128 + 4 * lane + (i & 3);
            if (e < left) p[e] = (uint8_t)(c[i >> 2] >> (8 * (i & 3)));
        }
    }
}

__device__ __forceinline__ void decode(const u32 (&c)[2], float scale, Oct &o)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        u32 h2;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((u16)(c[i >> 1] >> (16 * (i & 1)))));
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h2));
        o.x[2 * i] = __fmul_rn(f.x, scale);
        o.x[2 * i + 1] = __fmul_rn(f.y, scale);
    }
}

// A scaled value (below 256 in magnitude) moved to the E4M3 value above or below it in magnitude, to the one above with
// the probability of its fraction of the step between them: 16 random bits `b`, added (with half a unit more) below the
// three bits of the significand that stay. Under 2^-6 the steps are those of that binade, which adding 2^-6 brings about.
__device__ __forceinline__ float round_by_chance(float y, u32 b)
{
    const float a = fabsf(y), lift = a < 0x1p-6f ? 0x1p-6f : 0.0f;
    const u32 t = (__float_as_uint(__fadd_rn(a, lift)) + ((b << 4) | 8u)) & 0xFFF00000u;
    return copysignf(__fsub_rn(__uint_as_float(t), lift), y);
}

// Codes of the warp's block, and its scale. A power of two, so that scaling is exact. FLOOR: what is positive keeps a
// code of at least 1 (2^-9). The code is the nearest one, or with CHANCE one of the two around the value
// (`random`: two values' bits in a word). To nearest, a value that changes by less than half a step a call never moves: three
// bits of significand make that 3 to 6 %, and sqrt(beta2) is far nearer to 1. By chance, the mean moves as it should.
template <bool FLOOR, bool CHANCE>
__device__ __forceinline__ float encode(const Oct &o, u32 (&c)[2], const u32 (&random)[4])
{
    constexpr u32 INF = 0x7F800000u;
    u32 most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(o.x[i]) & 0x7FFFFFFFu);
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    const bool bad = most >= INF;           // (of the whole block, so the branches below are not divergent)
    if (bad) {                              // a value that is not finite must not become its neighbours' scale
        most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const u32 a = __float_as_uint(o.x[i]) & 0x7FFFFFFFu;
            most = max(most, a < INF ? a : 0u);
        }
        most = __reduce_max_sync(0xFFFFFFFFu, most);
    }
    const u32 e = (u32)max((int)(most >> 23) - 7, 1);
    const float inv = __uint_as_float((254u - e) << 23);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        u16 q[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float a = o.x[4 * j + 2 * i], b = o.x[4 * j + 2 * i + 1];
            float x = __fmul_rn(a, inv), y = __fmul_rn(b, inv);
            if (FLOOR) {
                if (a > 0.0f) x = fmaxf(x, 0x1p-9f);
                if (b > 0.0f) y = fmaxf(y, 0x1p-9f);
            }
            if (CHANCE) {
                x = round_by_chance(x, random[2 * j + i] & 0xFFFFu);
                y = round_by_chance(y, random[2 * j + i] >> 16);
            }
            // the second source goes to the low byte
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(q[i]) : "f"(y), "f"(x));
        }
        c[j] = __byte_perm(q[0], q[1], 0x5410);
        if (bad) {                          // infinity would saturate
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((__float_as_uint(o.x[4 * j + i]) & 0x7FFFFFFFu) >= INF) c[j] |= 0x7Fu << (8 * i);
        }
    }
    return __uint_as_float(e << 23);
}

// The gradient before clipping: one element, single fp32 operations.
__device__ __forceinline__ float total_gradient(const ListScalars &s, float gr, bool penalty, float w, float th, float lam)
{
    float g = __fmul_rn(s.grad_scale, gr);
    if (penalty) g = __fadd_rn(g, __fsub_rn(__fmul_rn(s.mu, __fsub_rn(w, th)), lam));
    return g;
}

// AdamW. Bytes per element: w 8, gradient 4 or 2, theta and lambda 8 with the penalty, moments 16
// (fp32) or 4 + 16/256 (8 bits), copy 2: bound by memory, and every byte is moved once.
// Measured on 135.9 M elements (shares of a plain copy's 6530 GB/s): fp32 gradients and moments with the penalty, 36 bytes
// an element, 773 us (0.97); bfloat16 gradients and copies with 8-bit moments, 16 bytes, 401 us (0.83, with 79
// instructions an element beside it) to nearest and 589 us by chance (the hash and two roundings more, bound by
// instructions). 1.9 M elements in 32 tensors: 9 us, a launch and one round of the CTAs.
template <int CAP, int GT, int STATES, bool PEN>
__global__ void __launch_bounds__(THREADS, adamw_ctas(STATES, PEN)) k_adamw(const __grid_constant__ ListParams<CAP> P)
{
    constexpr bool EIGHT = STATES != ST_32, CHANCE = STATES == ST_8_STOCHASTIC;
    const ListScalars &s = P.s;
    float coef = 1.0f;
    if (s.clip) {
        if (s.clip[2] == 0.0f) return;
        coef = s.clip[1];
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (u32 item = blockIdx.x; item < s.n_items; item += gridDim.x) {
        const int t = list_owner(P, item);
        const ListDesc &d = P.d[t];
        const u64 key = CHANCE ? mix64(s.key ^ (u64)(s.t0 + t)) : 0;
        const long long first = ((long long)(item - d.item0) * s.chunks * WARPS + warp) * LIST_CHUNK;
        for (int k = 0; k < s.chunks; ++k) {
            const long long e0 = first + (long long)k * WARPS * LIST_CHUNK, left = d.numel - e0;
            if (left <= 0) break;
            const bool vec = d.vec_ok && left >= LIST_CHUNK;
            const long long blk = e0 / LIST_CHUNK;
            // the warp's next chunk, of this item or of the CTA's next one where that is the same tensor's, is asked for
            // ahead: a line per lane, of w (8), the gradient (8 or 4), the codes (2 + 2). (Moments in 8 bits leave fewer
            // bytes in flight than those in 32: 456 -> 401 us on 135.9 M elements, and no register)
            const long long e1 = k + 1 < s.chunks ? e0 + WARPS * LIST_CHUNK : first + (long long)gridDim.x * s.chunks * (WARPS * LIST_CHUNK);
            if (EIGHT && d.numel - e1 >= LIST_CHUNK) {
                constexpr int GL = GT == GT_F32 ? 8 : 4;
                const char *p = lane < 8 ? (const char *)(d.w + e1) + lane * 128
                              : lane < 8 + GL ? (const char *)d.grad + e1 * (GT == GT_F32 ? 4 : 2) + (lane - 8) * 128
                              : lane < 10 + GL ? (const char *)d.m + e1 + (lane - 8 - GL) * 128 : (const char *)d.v + e1 + (lane - 10 - GL) * 128;
                if (lane < 12 + GL) asm volatile("prefetch.global.L2 [%0];" :: "l"(p));
            }
            Oct w = load_f32(d.w + e0, lane, left, vec);
            Oct g = load_grad<GT>(d.grad, e0, lane, left, vec);
            Oct th, lam, m, v;
            u32 cm[2], cv[2];
            float sm, sv;
            const bool has = PEN && d.theta != nullptr;
            if (PEN) {
                th = has ? load_f32(d.theta + e0, lane, left, vec) : Oct{};
                lam = has && d.lam ? load_f32(d.lam + e0, lane, left, vec) : Oct{};
            }
            if (EIGHT) {
                load_codes((const uint8_t *)d.m + e0, cm, lane, left, vec);
                load_codes((const uint8_t *)d.v + e0, cv, lane, left, vec);
                sm = d.m_scale[blk];
                sv = d.v_scale[blk];
            } else {
                m = load_f32((const float *)d.m + e0, lane, left, vec);
                v = load_f32((const float *)d.v + e0, lane, left, vec);
            }
            if (EIGHT) {
                decode(cm, sm, m);
                decode(cv, sv, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) v.x[i] = __fmul_rn(v.x[i], v.x[i]);
            }
            Oct root;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float gi = total_gradient(s, g.x[i], has, w.x[i], PEN ? th.x[i] : 0.0f, PEN ? lam.x[i] : 0.0f);
                gi = __fmul_rn(coef, gi);
                m.x[i] = __fadd_rn(__fmul_rn(s.beta1, m.x[i]), __fmul_rn(s.c1, gi));
                v.x[i] = __fadd_rn(__fmul_rn(s.beta2, v.x[i]), __fmul_rn(s.c2, __fmul_rn(gi, gi)));
                root.x[i] = __fsqrt_rn(v.x[i]);
                const float den = __fadd_rn(__fmul_rn(root.x[i], s.root_corr), s.eps);
                // (8 bits: nothing that is kept in codes comes from this quotient, and it saves instructions)
                const float quo = EIGHT ? __fdividef(m.x[i], den) : __fdiv_rn(m.x[i], den);
                w.x[i] = __fsub_rn(__fmul_rn(w.x[i], s.decay), __fmul_rn(s.step_size, quo));
            }
            store_f32(d.w + e0, w, lane, left, vec);
            if (d.w_h) store_copy(d.w_h + e0, w, s.copy_type, lane, left, vec);
            if (EIGHT) {
                // (places past the tensor's end hold 0 or NaN, which leave the block's scale alone)
                u32 rm[4] = {0, 0, 0, 0}, rv[4] = {0, 0, 0, 0};
                if (CHANCE) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {       // 64 bits for two elements: elements 2i and 2i + 1 of the pair of quads
                        const u64 z = mix64(key ^ (u64)((e0 + (i >> 1) * 128 + 4 * lane + 2 * (i & 1)) >> 1));
                        rm[i] = (u32)z;
                        rv[i] = (u32)(z >> 32);
                    }
                }
                sm = encode<false, CHANCE>(m, cm, rm);
                sv = encode<true, CHANCE>(root, cv, rv);
                store_codes((uint8_t *)d.m + e0, cm, lane, left, vec);
                store_codes((uint8_t *)d.v + e0, cv, lane, left, vec);
                __syncwarp();                       // every lane has read the old scales
                if (lane == 0) {
                    d.m_scale[blk] = sm;
                    d.v_scale[blk] = sv;
                }
            } else {
                store_f32((float *)d.m + e0, m, lane, left, vec);
                store_f32((float *)d.v + e0, v, lane, left, vec);
            }
        }
    }
}

// ------------------------------------------------------------------ norm
// Squares are summed in fp32 by groups of eight values, the groups in fp64. Bound by memory; the loads run a batch ahead
// of the sums (135.9 M values of bfloat16: 83 us without that, 53 us with it, 0.78 of a copy's rate; 58 tensors of
// 0.85 M values in all: 12.5 us, most of it the launch and the last CTA's sums). Each CTA takes a contiguous range of the
// work items and leaves one fp64 partial sum per tensor that it meets. CTA b's sum for tensor t goes to slot b + t: both only grow along the list, so no
// two pairs share a slot. The CTA that finishes last adds the slots of each tensor in order.
struct NormOut {
    double *slot;           // grid + T of them
    double *square;         // sums of squares of all tensors of the call
    u32 *done;              // CTAs finished; zero between launches
    float *norms;
    float *clip;
    int t0, T_all;          // this launch's first tensor; tensors of the call
    int last;               // this launch finishes the call
    float max_norm;
};

__device__ __forceinline__ double block_sum(double x, double *sh)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
    __syncthreads();
    double r = 0.0;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) r += sh[i];
    return r;
}

template <int CAP, int GT, bool PEN>
__global__ void __launch_bounds__(THREADS, 4) k_grad_norm(const __grid_constant__ ListParams<CAP> P, const NormOut N)
{
    __shared__ double sh[WARPS];
    __shared__ u32 s_last;
    const ListScalars &s = P.s;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const u32 n = s.n_items, G = gridDim.x;
    u32 item = (u32)((unsigned long long)blockIdx.x * n / G);
    const u32 end = (u32)((unsigned long long)(blockIdx.x + 1) * n / G);
    int t = item < end ? list_owner(P, item) : 0;
    while (item < end) {
        while (t + 1 < s.T && P.d[t + 1].item0 <= item) ++t;         // empty tensors own no item
        const ListDesc &d = P.d[t];
        const u32 stop = (t + 1 < s.T) ? min(end, P.d[t + 1].item0) : end;
        double sum = 0.0;
        const bool has_th = PEN && d.theta != nullptr, has_lam = has_th && d.lam != nullptr;
        auto add = [&](const Oct &g) {
            float part = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) part = fmaf(g.x[i], g.x[i], part);
            if (part >= 0x1p-90f && part <= 0x1p120f) sum += (double)part;
            else {                  // squares beyond what fp32 holds on either side, or zeros
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = fma((double)g.x[i], (double)g.x[i], sum);
            }
        };
        // one step: a chunk per warp. Chunks that exist as a whole, of aligned tensors without a penalty, are loaded UN at a
        // time, a batch ahead of the one that is summed
        long long c = (long long)(item - d.item0) * s.chunks;
        const long long c1 = (long long)(stop - d.item0) * s.chunks;
        if (!PEN && d.vec_ok) {
            constexpr int UN = GT == GT_F32 ? 2 : 4;
            const long long whole = min(c1, d.numel / (WARPS * LIST_CHUNK));       // steps that every warp has a whole chunk of
            const long long batches = max(0ll, whole - c) / UN;
            Raw<GT> r0[UN], r1[UN];
            const char *p = (const char *)d.grad + (c * WARPS + warp) * (LIST_CHUNK * (GT == GT_F32 ? 4 : 2));
            auto load = [&](Raw<GT> (&r)[UN]) {
#pragma unroll
                for (int q = 0; q < UN; ++q) {
                    r[q].load(p, lane);
                    p += WARPS * LIST_CHUNK * (GT == GT_F32 ? 4 : 2);
                }
            };
            auto use = [&](const Raw<GT> (&r)[UN]) {
#pragma unroll
                for (int q = 0; q < UN; ++q) {
                    Oct g = r[q].widened();
#pragma unroll
                    for (int i = 0; i < 8; ++i) g.x[i] = __fmul_rn(s.grad_scale, g.x[i]);
                    add(g);
                }
            };
            if (batches > 0) load(r0);
#pragma unroll 1
            for (long long i = 0; i < batches; i += 2) {
                if (i + 1 < batches) load(r1);
                use(r0);
                if (i + 2 < batches) load(r0);
                if (i + 1 < batches) use(r1);
            }
            c += batches * UN;
        }
#pragma unroll 1
        for (; c < c1; ++c) {
            const long long e0 = (c * WARPS + warp) * LIST_CHUNK, left = d.numel - e0;
            if (left <= 0) continue;
            const bool vec = d.vec_ok && left >= LIST_CHUNK;
            Oct g = load_grad<GT>(d.grad, e0, lane, left, vec), w, th, lam;
            if (PEN) {
                w = has_th ? load_f32(d.w + e0, lane, left, vec) : Oct{};
                th = has_th ? load_f32(d.theta + e0, lane, left, vec) : Oct{};
                lam = has_lam ? load_f32(d.lam + e0, lane, left, vec) : Oct{};
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                g.x[i] = total_gradient(s, g.x[i], has_th, PEN ? w.x[i] : 0.0f, PEN ? th.x[i] : 0.0f, PEN ? lam.x[i] : 0.0f);
            add(g);
        }
        sum = block_sum(sum, sh);
        if (threadIdx.x == 0) N.slot[blockIdx.x + t] = sum;
        item = stop;
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) s_last = atomicAdd(N.done, 1u) == G - 1;
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    // all slots at once (some are nobody's and hold what they held), then each tensor's in order
    __shared__ double slots[NORM_GRID_MAX + CAP];
    for (u32 i = threadIdx.x; i < G + (u32)s.T - 1; i += THREADS) slots[i] = __ldcg(N.slot + i);
    __syncthreads();
    for (int q = warp; q < s.T; q += WARPS) {
        const u32 i0 = P.d[q].item0, i1 = q + 1 < s.T ? P.d[q + 1].item0 : n;
        double sum = 0.0;
        if (i1 > i0) {
            const u32 b0 = (u32)((((unsigned long long)i0 + 1) * G - 1) / n), b1 = (u32)(((unsigned long long)i1 * G - 1) / n);
            for (u32 b = b0 + lane; b <= b1; b += 32) sum += slots[b + q];
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        if (lane == 0) {
            N.square[N.t0 + q] = sum;
            if (N.norms) N.norms[N.t0 + q] = (float)sqrt(sum);
        }
    }
    __syncthreads();
    if (N.last) {
        double sum = 0.0;
        for (int q = threadIdx.x; q < N.T_all; q += THREADS) sum += N.square[q];
        sum = block_sum(sum, sh);
        if (threadIdx.x == 0) {
            const float norm = (float)sqrt(sum);
            const bool fine = (__float_as_uint(norm) & 0x7FFFFFFFu) < 0x7F800000u;
            N.clip[0] = norm;
            N.clip[1] = N.max_norm > 0.0f && fine ? fminf(1.0f, __fdiv_rn(N.max_norm, __fadd_rn(norm, 1e-6f))) : 1.0f;
            N.clip[2] = fine ? 1.0f : 0.0f;
            N.clip[3] = 0.0f;
        }
    }
    if (threadIdx.x == 0) *N.done = 0;
}

}  // namespace cs
