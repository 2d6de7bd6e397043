// Low-rank adapters of many requests beside one shared projection.
//
// With S the matrix that shrinks a row to `rank` numbers and E the one that expands them again
// (forward: S = A, E = B; backward: S = B^T, E = A^T), both directions are the same two products:
//
//     h = S * src        [rank]        dst <- dst + E * (factor * h)
//
// k_adapter does both in one launch. A tile is up to TM rows of one adapter, from one request or from
// several; a thread-block cluster works on it. Each CTA of the cluster contracts its part of the source
// columns, the CTAs add their partial h over distributed shared memory, and each then expands its part
// of the destination columns, whose first values are already on their way. src is read once, dst once
// and written once, h never makes a trip through global memory in between.
//
// The arithmetic is small (2 * rank operations per source and destination element), so the
// kernels are bound by memory up to ranks of 64 or so; the row kernel's products run on the warp-level matrix
// instruction, whose operands are loaded from global memory straight into the registers that it wants them in: the
// order of the terms of a sum is free, so each lane takes 16 neighbouring bytes of a row for two steps of the
// product, of src and of the matrix alike. No shared memory and no barrier stand in its two loops. (Staged through a
// ring in shared memory, the same products were 1.3 to 2 times slower: two barriers' worth of latency per chunk, and
// most instructions spent on copies.)
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <type_traits>
#include "common.cuh"

namespace cs {

typedef unsigned short u16;

constexpr int AD_BLOB = 3840;                // bytes of lists in the kernel parameters
constexpr int AD_MAX_RANK = 128;
constexpr int AD_MAX_CLUSTER = 8;
constexpr int AD_MAX_WIDTH = 1 << 22;        // of x and y: places in A are 32-bit offsets (2^22 * 128 ranks * 4 bytes = 2^31)
constexpr int AD_WG_ROWS = 64;               // rows of a tile of the weight gradients

struct AdapterRun {                          // rows of an adapter that follow one another
    int first;                               // the first of them
    int before;                              // the adapter's rows ahead of it
};

struct AdapterEntry {                        // an adapter as k_adapter sees it
    const void *shrink;
    const void *expand;
    float scale;
    int n_rows;
    int tile0;                               // its first tile
    u16 run0, n_runs;                        // its rows
    u16 rank, pad;
    int ld_s, ld_e;                          // row strides: shrink [rank][source columns], expand [destination columns][rank]
};
static_assert(sizeof(AdapterEntry) == 48, "packed into the parameters");

struct AdapterParams {
    const void *src;
    void *dst;                               // NULL: nothing is expanded
    float *h;                                // h (forward) or scale * S src (backward); NULL: not kept
    long long ld_src, ld_dst, ld_h;
    long long width_src, width_dst;
    int vec_src, vec_dst;
    int n_entries;
    int splits;                              // clusters that share a tile's destination columns (each forms all of h)
    int scale_h;                             // 1 (backward): h is scale * S src, and the expansion takes no factor
    int pad;
    u32 blob[AD_BLOB / 4];                   // entries, runs
};
static_assert(sizeof(AdapterParams) <= 4096, "kernel parameters");

// Row i of an adapter with these runs.
__device__ __forceinline__ int adapter_row(const AdapterRun *runs, int n, int i)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (runs[mid].before <= i) lo = mid; else hi = mid - 1;
    }
    return runs[lo].first + (i - runs[lo].before);
}

// ------------------------------------------------------------------ types
template <class T> struct AdType {           // 16-bit types
    static constexpr int E = 2, KSTEP = 16;              // bytes; depth of a product step
    static constexpr int PARTS = 2;                      // 16-bit parts of an fp32 operand of the expansion
};
template <> struct AdType<float> {
    static constexpr int E = 4, KSTEP = 8;
    static constexpr int PARTS = 1;
};

__device__ __forceinline__ u32 smem_u32(const void *p) { return (u32)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void cp16(u32 dst, const void *src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp8(u32 dst, const void *src, int bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" :: "r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp4(u32 dst, const void *src, int bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

__device__ __forceinline__ void st_shared16(u32 dst, uint4 v)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(dst), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// 16 bytes of a row into shared memory, the first `n` (0 to 16) of them exist (the rest become zero). V: the
// accesses that every row allows, 16 or 8 bytes; 0: `vec` says it. `any`: an address that may be formed where
// nothing exists.
template <int V>
__device__ __forceinline__ void copy_unit(u32 dst, const char *src, const char *any, int n, int vec)
{
    if (V == 16) {
        cp16(dst, n ? src : any, n);
    } else if (V == 8 || vec >= 8) {
        const int m = max(n - 8, 0);
        cp8(dst, n ? src : any, min(n, 8));
        cp8(dst + 8, m ? src + 8 : any, m);
    } else if (vec == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int m = min(max(n - 4 * i, 0), 4);
            cp4(dst + 4 * i, m ? src + 4 * i : any, m);
        }
    } else {
        u32 w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (n > 2 * i) w[i >> 1] |= (u32) * reinterpret_cast<const u16 *>(src + 2 * i) << (16 * (i & 1));
        st_shared16(dst, make_uint4(w[0], w[1], w[2], w[3]));
    }
}

__device__ __forceinline__ void ldsm4(u32 (&r)[4], u32 addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(u32 (&r)[4], u32 addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ float lds_f32(u32 addr)
{
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
// Operand fragments of one product step (16 x KSTEP times KSTEP x 8).
template <class T> struct FragA { u32 r[4]; };
template <class T> struct FragB { u32 r[2]; };
template <> struct FragA<float> { u32 hi[4], lo[4]; };       // two TF32 parts: 22 bits of the operand
template <> struct FragB<float> { u32 hi[2], lo[2]; };

// (the instruction reads the upper 19 bits of an operand: the second part, at most 2^-12 of the value, is cut there.
// No number stays one: its rest is no number. From 2^128 - 2^116 on the first part is infinite and the second the other
// infinity; to cut there instead of rounding costs two instructions a value and 15 % of a call.)
__device__ __forceinline__ void split_tf32(float x, u32 &hi, u32 &lo)
{
    hi = (__float_as_uint(x) + 0x1000u) & 0xFFFFE000u;
    lo = __float_as_uint(x - __uint_as_float(hi));
}

__device__ __forceinline__ void mma_step(float (&c)[4], const FragA<__nv_bfloat16> &a, const FragB<__nv_bfloat16> &b)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a.r[0]), "r"(a.r[1]), "r"(a.r[2]), "r"(a.r[3]), "r"(b.r[0]), "r"(b.r[1]));
}
__device__ __forceinline__ void mma_step(float (&c)[4], const FragA<__half> &a, const FragB<__half> &b)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a.r[0]), "r"(a.r[1]), "r"(a.r[2]), "r"(a.r[3]), "r"(b.r[0]), "r"(b.r[1]));
}
// The same on a sum that starts at zero.
__device__ __forceinline__ void mma_first(float (&c)[4], const FragA<__nv_bfloat16> &a, const FragB<__nv_bfloat16> &b)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a.r[0]), "r"(a.r[1]), "r"(a.r[2]), "r"(a.r[3]), "r"(b.r[0]), "r"(b.r[1]), "f"(0.0f));
}
__device__ __forceinline__ void mma_first(float (&c)[4], const FragA<__half> &a, const FragB<__half> &b)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a.r[0]), "r"(a.r[1]), "r"(a.r[2]), "r"(a.r[3]), "r"(b.r[0]), "r"(b.r[1]), "f"(0.0f));
}
__device__ __forceinline__ void mma_tf32(float (&c)[4], const u32 (&a)[4], const u32 (&b)[2])
{
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ void mma_step(float (&c)[4], const FragA<float> &a, const FragB<float> &b)
{
    mma_tf32(c, a.lo, b.hi);        // small terms first; lo * lo lies below fp32
    mma_tf32(c, a.hi, b.lo);
    mma_tf32(c, a.hi, b.hi);
}
__device__ __forceinline__ void mma_first(float (&c)[4], const FragA<float> &a, const FragB<float> &b)
{
    c[0] = c[1] = c[2] = c[3] = 0.0f;
    mma_step(c, a, b);
}

// A operand from [k][m] (its transpose lies in memory).
template <class T>
__device__ __forceinline__ void load_a_t(FragA<T> &f, u32 base, int stride, int lane)
{
    const int q = lane >> 3;
    ldsm4t(f.r, base + ((q >> 1) * 8 + (lane & 7)) * stride + (q & 1) * 16);
}
__device__ __forceinline__ void load_a_t(FragA<float> &f, u32 base, int stride, int lane)
{
    const u32 p = base + (lane & 3) * stride + (lane >> 2) * 4;
    split_tf32(lds_f32(p), f.hi[0], f.lo[0]);
    split_tf32(lds_f32(p + 32), f.hi[1], f.lo[1]);
    split_tf32(lds_f32(p + 4 * stride), f.hi[2], f.lo[2]);
    split_tf32(lds_f32(p + 4 * stride + 32), f.hi[3], f.lo[3]);
}
// B operands of two neighbouring 8-column tiles from [k][n].
template <class T>
__device__ __forceinline__ void load_b2_t(FragB<T> (&f)[2], u32 base, int stride, int lane)
{
    u32 r[4];
    const int q = lane >> 3;
    ldsm4t(r, base + ((q & 1) * 8 + (lane & 7)) * stride + (q >> 1) * 16);
    f[0].r[0] = r[0]; f[0].r[1] = r[1]; f[1].r[0] = r[2]; f[1].r[1] = r[3];
}
__device__ __forceinline__ void load_b2_t(FragB<float> (&f)[2], u32 base, int stride, int lane)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const u32 p = base + (lane & 3) * stride + (i * 8 + (lane >> 2)) * 4;
        split_tf32(lds_f32(p), f[i].hi[0], f[i].lo[0]);
        split_tf32(lds_f32(p + 4 * stride), f[i].hi[1], f[i].lo[1]);
    }
}

// 16-bit parts of an fp32 value: hi + lo (+ lo2) holds 16 (24) bits of it in bfloat16, 22 in binary16. One that is
// not finite has no further parts.
template <class T, int PARTS>
__device__ __forceinline__ void split16(float x, u16 (&p)[PARTS])
{
    const bool fine = (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        const T q = (T)x;
        p[i] = *reinterpret_cast<const u16 *>(&q);
        x = fine ? x - (float)q : 0.0f;
    }
}

// Power of two whose inverse brings `most` into [2^13, 2^14): as far up as sums allow, since binary16 ends 2^-24 above zero. (1
// where `most` is not finite; values below 2^-113 stay as far below 2^13.)
__device__ __forceinline__ float pow2_unit(float most)
{
    const u32 e = (__float_as_uint(most) >> 23) & 0xFFu;
    return e == 255u ? 1.0f : __uint_as_float((max(e, 14u) - 13u) << 23);
}
__device__ __forceinline__ float pow2_inverse(float p) { return __uint_as_float((254u << 23) - __float_as_uint(p)); }

// ------------------------------------------------------------------ cluster
__device__ __forceinline__ u32 cluster_rank() { u32 r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ u32 cluster_size() { u32 r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float4 ld_cluster(u32 addr, u32 rank)
{
    u32 a;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}

// ------------------------------------------------------------------ fragments straight from rows
// Step s (0 or 1) of a block of 4 * (16 / E) columns: lane t of a quad holds 16 bytes of each row, words 2s and 2s + 1 of
// them are its share of the step's depth. In both operands alike, so the permutation of the depth drops out.
template <class T>
__device__ __forceinline__ void frag_a(FragA<T> &f, const uint4 &up, const uint4 &low, int s)
{
    f.r[0] = s ? up.z : up.x; f.r[1] = s ? low.z : low.x;
    f.r[2] = s ? up.w : up.y; f.r[3] = s ? low.w : low.y;
}
__device__ __forceinline__ void frag_a(FragA<float> &f, const uint4 &up, const uint4 &low, int s)
{
    split_tf32(__uint_as_float(s ? up.z : up.x), f.hi[0], f.lo[0]);
    split_tf32(__uint_as_float(s ? low.z : low.x), f.hi[1], f.lo[1]);
    split_tf32(__uint_as_float(s ? up.w : up.y), f.hi[2], f.lo[2]);
    split_tf32(__uint_as_float(s ? low.w : low.y), f.hi[3], f.lo[3]);
}
template <class T>
__device__ __forceinline__ void frag_b(FragB<T> &f, u32 w0, u32 w1)
{
    f.r[0] = w0; f.r[1] = w1;
}
__device__ __forceinline__ void frag_b(FragB<float> &f, u32 w0, u32 w1)
{
    split_tf32(__uint_as_float(w0), f.hi[0], f.lo[0]);
    split_tf32(__uint_as_float(w1), f.hi[1], f.lo[1]);
}
template <class T>
__device__ __forceinline__ void frag_h(FragA<T> &f, uint2 up, uint2 low)
{
    f.r[0] = up.x; f.r[1] = low.x; f.r[2] = up.y; f.r[3] = low.y;
}
__device__ __forceinline__ void frag_h(FragA<float> &f, uint2 up, uint2 low)
{
    split_tf32(__uint_as_float(up.x), f.hi[0], f.lo[0]);
    split_tf32(__uint_as_float(low.x), f.hi[1], f.lo[1]);
    split_tf32(__uint_as_float(up.y), f.hi[2], f.lo[2]);
    split_tf32(__uint_as_float(low.y), f.hi[3], f.lo[3]);
}

// 16 bytes of a row. V: the access that every row allows, 16 or 8 bytes; 0: value by value. STREAM: read once,
// not worth a place in the L1 cache, where A and B are shared by the warps.
template <int V, int E, bool STREAM>
__device__ __forceinline__ uint4 load_unit(const char *p)
{
    uint4 r;
    if (V == 16) {
        if (STREAM) asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
        else r = *reinterpret_cast<const uint4 *>(p);
    } else if (V == 8) {
        const uint2 a = reinterpret_cast<const uint2 *>(p)[0], b = reinterpret_cast<const uint2 *>(p)[1];
        r = make_uint4(a.x, a.y, b.x, b.y);
    } else if (E == 4) {
        const u32 *q = reinterpret_cast<const u32 *>(p);
        r = make_uint4(q[0], q[1], q[2], q[3]);
    } else {
        const u16 *q = reinterpret_cast<const u16 *>(p);
        r = make_uint4(q[0] | (u32)q[1] << 16, q[2] | (u32)q[3] << 16, q[4] | (u32)q[5] << 16, q[6] | (u32)q[7] << 16);
    }
    return r;
}
// The first n values of it; the others are zero.
template <int E>
__device__ __noinline__ uint4 load_some(const char *p, int n)
{
    u32 w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16 / E; ++i)
        if (i < n) {
            if (E == 4) w[i] = reinterpret_cast<const u32 *>(p)[i];
            else w[i >> 1] |= (u32)reinterpret_cast<const u16 *>(p)[i] << (16 * (i & 1));
        }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Sixteen bytes of destination values plus factor times a lane's accumulators, rounded once.
__device__ __forceinline__ void unpack2(u32 w, float &lo, float &hi, __nv_bfloat16)
{
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xFFFF0000u);
}
__device__ __forceinline__ void unpack2(u32 w, float &lo, float &hi, __half)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    lo = f.x;
    hi = f.y;
}
__device__ __forceinline__ u32 pack2(float lo, float hi, __nv_bfloat16)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const u32 *>(&v);
}
__device__ __forceinline__ u32 pack2(float lo, float hi, __half)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const u32 *>(&v);
}
template <class T, int NT>
__device__ __forceinline__ uint4 add_unit(const uint4 &old, const float (&d)[NT][4], int half, float factor)
{
    const u32 o[4] = {old.x, old.y, old.z, old.w};
    u32 w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 2) {
            float lo, hi;
            unpack2(o[j], lo, hi, T());
            w[j] = pack2(fmaf(factor, d[j][2 * half], lo), fmaf(factor, d[j][2 * half + 1], hi), T());
        } else {
            w[j] = __float_as_uint(fmaf(factor, d[j >> 1][2 * half + (j & 1)], __uint_as_float(o[j])));
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int V, int E>
__device__ __forceinline__ void store_unit(char *p, const uint4 &v, int n)
{
    if (V == 16 && n == 16 / E) *reinterpret_cast<uint4 *>(p) = v;
    else if (V == 8 && n == 16 / E) {
        reinterpret_cast<uint2 *>(p)[0] = make_uint2(v.x, v.y);
        reinterpret_cast<uint2 *>(p)[1] = make_uint2(v.z, v.w);
    } else {
        const u32 w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 16 / E; ++e)
            if (e < n) {
                if (E == 4) reinterpret_cast<u32 *>(p)[e] = w[e];
                else reinterpret_cast<u16 *>(p)[e] = (u16)(w[e >> 1] >> (16 * (e & 1)));
            }
    }
}

// ------------------------------------------------------------------ geometry
// A warp takes 16 rows; the RG warps above one another cover the tile, the KW side by side share its columns.
template <class T, int TM, int RP>
struct AdGeom {
    static constexpr int E = AdType<T>::E, U = 16 / E;               // bytes of a value; values of a lane's unit
    static constexpr int RG = TM / 16, KW = WARPS / RG;
    static constexpr int KB = 4 * U, NT = U / 2;                     // columns of a block; 8-column product tiles of one
    static constexpr int NB = RP <= 16 ? 2 : 1;                      // source blocks of a step of the first loop
    // A and B, too, are loaded a step ahead; else half a step. (Short tiles, a decoding step's, are bound by latency
    // alone and leave registers to spare)
    static constexpr bool AHEAD = RP <= 32 || (TM == 16 && RP == 64);
    // Tiles of the rank whose sums of a step are kept apart at a time: all, or two where registers are short (four at 64
    // ranks spill 300 to 600 bytes, two under 140)
    static constexpr int APART = RP <= 32 ? RP / 8 : 2;
    static constexpr int HP_STRIDE = RP + 4;                         // floats
    static constexpr int HP = (KW > 1 ? KW / 2 : 1) * TM * HP_STRIDE * 4;    // partial sums
    static constexpr int HO_STRIDE = RP * E + (RP * E == 32 ? 0 : 32);       // operand of the expansion: four rows meet all banks
    static constexpr int HO = TM * HO_STRIDE * AdType<T>::PARTS;
    static constexpr int SMEM = HP + HO + TM * 8;
    static constexpr int CTAS = RP <= 32 || (TM == 64 && RP == 64) ? 2 : 1;                    // resident on an SM, at least
    static_assert(HP % 16 == 0 && HO % 16 == 0 && SMEM <= 227 * 1024, "shared memory");
};

// Measured: 6011 rows of 9216 -> 4096, rank 16, bf16: 52 us, 0.57 of a copy's rate; a load of 16 bytes a lane touches 8
// rows, so L1 looks up 8 lines for it, and that is the bound. 700 rows of 1500 -> 33278, fp32, accesses of 8 bytes: 69 us
// (0.44). Backward, 8192 rows of 4096 and 4096 columns: 43 us (floor 31). Decoding, 64 rows of 4096 -> 4096, ranks to
// 64, fp16: 11 us, the latency of few warps' dependent instructions.
template <class T, int TM, int RP, int V>
__global__ void __launch_bounds__(THREADS, AdGeom<T, TM, RP>::CTAS) k_adapter(const __grid_constant__ AdapterParams P)
{
    using G = AdGeom<T, TM, RP>;
    constexpr int E = G::E, U = G::U, NT = G::NT, NB = G::NB, KB = G::KB, KW = G::KW, KSTEP = AdType<T>::KSTEP, PARTS = AdType<T>::PARTS;
    constexpr int JT = RP / 8, ST = RP / KSTEP;                      // tiles and steps of the rank
    constexpr int BLOCK = KB * E;                                    // bytes of a block: 64
    extern __shared__ __align__(128) char sm[];
    float *hp = reinterpret_cast<float *>(sm);
    char *ho = sm + G::HP;
    int *srow = reinterpret_cast<int *>(ho + G::HO);
    float *sfac = reinterpret_cast<float *>(srow + TM);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
    const int rg = warp / KW, kw = warp % KW;
    const int C = (int)cluster_size(), c_rank = (int)cluster_rank();

    const AdapterEntry *entries = reinterpret_cast<const AdapterEntry *>(P.blob);
    const AdapterRun *runs = reinterpret_cast<const AdapterRun *>(entries + P.n_entries);
    const int tile = (int)blockIdx.x / (C * P.splits), split = (int)blockIdx.x / C % P.splits;
    // the tile's adapter: entries are in order of their first tiles (all looked at together: one load's latency)
    int which = -1;
    for (int e = lane; e - lane < P.n_entries; e += 32) which += __popc(__ballot_sync(0xFFFFFFFFu, e < P.n_entries && entries[e].tile0 <= tile));
    const AdapterEntry &ent = entries[which];
    const int row0 = (tile - ent.tile0) * TM, count = min(TM, ent.n_rows - row0), rank = ent.rank, r16 = (rank + 15) & ~15;
    // (places without a row take the tile's first: what they yield is dropped)
    if (tid < TM) srow[tid] = adapter_row(runs + ent.run0, ent.n_runs, row0 + (tid < count ? tid : 0));
    __syncthreads();

    const int ws = (int)P.width_src, wd = (int)P.width_dst;          // (below 2^31)
    const int KBT = (ws + KB - 1) / KB, NBT = P.dst ? (wd + KB - 1) / KB : 0;
    // this warp's source blocks, and its destination blocks (kw, kw + KW, ... of the CTA's)
    const int kparts = C * KW, kpart = c_rank * KW + kw;
    const int KST = (KBT + NB - 1) / NB;                             // (whole steps of NB blocks, but at the very end)
    const int kb0 = NB * (int)((long long)kpart * KST / kparts), kb1 = min(KBT, NB * (int)((long long)(kpart + 1) * KST / kparts));
    const int part = split * C + c_rank, parts = C * P.splits;
    const int nb0 = (int)((long long)part * NBT / parts) + kw, nb1 = (int)((long long)(part + 1) * NBT / parts);
    const char *px[2];
    char *py[2];
    bool live[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const long long row = srow[rg * 16 + g + 8 * h];
        px[h] = (const char *)P.src + (row * P.ld_src + t4 * U) * E + (long long)kb0 * BLOCK;
        py[h] = (char *)P.dst + (row * P.ld_dst + t4 * U) * E + (long long)nb0 * BLOCK;
        live[h] = rg * 16 + g + 8 * h < count;
    }

    // ---- shrink: this warp's share of h. The blocks that exist as a whole go through two sets of registers in turn
    float acc[JT][4];
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[j][q] = 0.0f;
    struct SrcX { uint4 x[NB][2]; };
    constexpr int JH = G::AHEAD ? JT : JT / 2;              // tiles of the rank that are loaded at a time
    struct SrcW { uint4 w[NB][JH]; };
    // rows of S past the rank are read as its last one: what they yield is dropped
    const char *pw = (const char *)ent.shrink + (long long)kb0 * BLOCK + t4 * 16;
    u32 w_off[JT];
#pragma unroll
    for (int j = 0; j < JT; ++j) w_off[j] = (u32)min(8 * j + g, rank - 1) * (u32)(ent.ld_s * E);
    auto load_x = [&](SrcX &s) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int b = 0; b < NB; ++b) s.x[b][h] = load_unit<V, E, true>(px[h] + b * BLOCK);
            px[h] += NB * BLOCK;
        }
    };
    auto load_w = [&](SrcW &s, int j0) {
#pragma unroll
        for (int j = 0; j < JH; ++j) {
            if (j0 + j >= 2 && (j0 + j) * 8 >= r16) break;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                // (a matrix laid out anew allows 16 bytes; A as it is where V is 8, only 8)
                const char *p = pw + w_off[j0 + j] + b * BLOCK;
                if (V != 8 || P.scale_h) s.w[b][j] = load_unit<16, E, false>(p);
                else s.w[b][j] = load_unit<8, E, false>(p);
            }
        }
        if (j0 + JH == JT) pw += NB * BLOCK;
    };
    // The matrix instruction truncates its sums: those of a step (4 products in a row, fp32: 12) are kept apart and added with
    // rounding, or the loss would grow with the width (9216 columns of one sign, rank 64, fp32: 1.2e-5 of the sum, so 9e-8; the time
    // of a call changes by -3 to 3 %). JG tiles at a time, as registers allow.
    auto multiply = [&](const SrcX &x, const SrcW &w, int blocks, int j0) {
        constexpr int JG = G::APART < JH ? G::APART : JH;
#pragma unroll
        for (int jg = 0; jg < JH; jg += JG) {
            if (j0 + jg >= 2 && (j0 + jg) * 8 >= r16) break;
            float d[JG][4];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (b >= blocks) break;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    FragA<T> a;
                    frag_a(a, x.x[b][0], x.x[b][1], t);
#pragma unroll
                    for (int j = jg; j < jg + JG; ++j) {
                        if (j0 + j >= 2 && (j0 + j) * 8 >= r16) break;
                        FragB<T> f;
                        frag_b(f, t ? w.w[b][j].z : w.w[b][j].x, t ? w.w[b][j].w : w.w[b][j].y);
                        if (b == 0 && t == 0) mma_first(d[j - jg], a, f);
                        else mma_step(d[j - jg], a, f);
                    }
                }
            }
#pragma unroll
            for (int j = jg; j < jg + JG; ++j) {
                if (j0 + j >= 2 && (j0 + j) * 8 >= r16) break;
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[j0 + j][q] += d[j - jg][q];
            }
        }
    };
    {
        const int steps = max(0, min(kb1, ws / KB) - kb0) / NB;
        SrcX x0, x1;
        SrcW w0, w1;
        if (steps > 0) load_x(x0);
        pdl_wait();             // A and B may have been laid out by the kernel ahead
        pdl_launch_dependents();
        if (steps > 0) load_w(w0, 0);
        if constexpr (G::AHEAD) {
#pragma unroll 1
            for (int i = 0; i < steps; i += 2) {
                if (i + 1 < steps) {
                    load_x(x1);
                    load_w(w1, 0);
                }
                multiply(x0, w0, NB, 0);
                if (i + 2 < steps) {
                    load_x(x0);
                    load_w(w0, 0);
                }
                if (i + 1 < steps) multiply(x1, w1, NB, 0);
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < steps; i += 2) {
                load_w(w1, JH);
                if (i + 1 < steps) load_x(x1);
                multiply(x0, w0, NB, 0);
                if (i + 1 < steps) load_w(w0, 0);
                multiply(x0, w1, NB, JH);
                if (i + 1 < steps) {
                    load_w(w1, JH);
                    if (i + 2 < steps) load_x(x0);
                    multiply(x1, w0, NB, 0);
                    if (i + 2 < steps) load_w(w0, 0);
                    multiply(x1, w1, NB, JH);
                }
            }
        }
        // what is left: at most NB blocks, the last of them perhaps in part
#pragma unroll 1
        for (int kb = kb0 + steps * NB; kb < kb1; ++kb) {
            const int n = min(max(ws - kb * KB - t4 * U, 0), U);
            const bool whole = (kb + 1) * KB <= ws;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                x0.x[0][h] = whole ? load_unit<V, E, true>(px[h]) : load_some<E>(px[h], n);
                px[h] += BLOCK;
            }
#pragma unroll
            for (int j0 = 0; j0 < JT; j0 += JH) {
#pragma unroll
                for (int j = 0; j < JH; ++j) {
                    if (j0 + j >= 2 && (j0 + j) * 8 >= r16) break;
                    w0.w[0][j] = whole ? load_unit<8, E, false>(pw + w_off[j0 + j]) : load_some<E>(pw + w_off[j0 + j], n);
                }
                multiply(x0, w0, 1, j0);
            }
            pw += BLOCK;
        }
    }
    // ---- the first destination block sets out. The accumulator columns of tile j are columns 2j, 2j + 1 of every lane's U:
    // that is the column of B which this lane's 8-column index g stands for
    struct DstY { uint4 y[2]; };
    constexpr int SH = G::AHEAD ? ST : ST / 2;              // steps of the rank that are loaded at a time
    struct DstB { uint2 b[SH][NT]; };
    const int bcol = (g >> 1) * U + (g & 1);
    const char *pb = (const char *)ent.expand + (((long long)nb0 * KB + bcol) * ent.ld_e + t4 * (KSTEP / 4)) * E;
    const long long b_next = (long long)KW * KB * ent.ld_e * E;
    const u32 b_pair = 2u * (u32)ent.ld_e * E;
    // a lane holds a quad of ranks per step; those past the end of a row are read as zeros (ranks are whole quads here)
    u32 b_there = 0;
#pragma unroll
    for (int s = 0; s < ST; ++s)
        if (s * KSTEP + t4 * (KSTEP / 4) < rank) b_there |= 1u << s;
    // (of a block that exists in part, columns past the end are read as the last one)
    auto load_b = [&](DstB &d, int s0, int last) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const char *p = pb + (last < KB ? (long long)(min(bcol + 2 * j, last) - bcol) * ent.ld_e * E : (long long)(j * b_pair));
#pragma unroll
            for (int s = 0; s < SH; ++s) {
                if (s0 + s && (s0 + s) * KSTEP >= r16) break;
                d.b[s][j] = (b_there >> (s0 + s) & 1) ? *reinterpret_cast<const uint2 *>(p + (s0 + s) * KSTEP * E) : make_uint2(0, 0);
            }
        }
        if (s0 + SH == ST) pb += b_next;
    };
    auto load_y = [&](DstY &d) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            d.y[h] = load_unit<V, E, true>(py[h]);
            py[h] += KW * BLOCK;
        }
    };
    const int blocks = max(0, min(nb1, wd / KB) - nb0 + KW - 1) / KW;          // that exist as a whole
    DstY y0, y1;
    DstB b0;
    if (blocks > 0) {
        load_y(y0);
        load_b(b0, 0, KB);
    }
    // ---- the warps of a row group add up, the upper half handing its sums to the lower
    auto spot = [&](int slot, int j, int half) { return hp + ((slot * TM + rg * 16 + g + 8 * half) * G::HP_STRIDE + j * 8 + 2 * t4); };
    auto put = [&](int slot) {
#pragma unroll
        for (int j = 0; j < JT; ++j) {
            if (j * 8 >= r16) break;
            *reinterpret_cast<float2 *>(spot(slot, j, 0)) = make_float2(acc[j][0], acc[j][1]);
            *reinterpret_cast<float2 *>(spot(slot, j, 1)) = make_float2(acc[j][2], acc[j][3]);
        }
    };
#pragma unroll 1
    for (int w = KW / 2; w >= 1; w >>= 1) {
        if (kw >= w && kw < 2 * w) put(kw - w);
        __syncthreads();
        if (kw < w) {
#pragma unroll
            for (int j = 0; j < JT; ++j) {
                if (j * 8 >= r16) break;
                const float2 p = *reinterpret_cast<const float2 *>(spot(kw, j, 0)), q = *reinterpret_cast<const float2 *>(spot(kw, j, 1));
                acc[j][0] += p.x; acc[j][1] += p.y; acc[j][2] += q.x; acc[j][3] += q.y;
            }
        }
        __syncthreads();
    }
    if (kw == 0) put(0);
    // ---- the CTAs of the cluster add up, in order of their rank; every one of them needs all of h
    cluster_arrive();
    cluster_wait();
    const float factor = P.scale_h ? 1.0f : ent.scale;
    {
        constexpr int TPR = THREADS / TM;                    // threads of a row
        constexpr int QT = (RP / 4 + TPR - 1) / TPR;         // quads of a thread
        const int r = tid / TPR, sub = tid % TPR;
        const float f = P.scale_h ? ent.scale : 1.0f;
        float4 v[QT];
        float most = 0.0f;
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            const int c = 4 * (q * TPR + sub);
            v[q] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (c < r16) {
                const u32 at = smem_u32(hp + r * G::HP_STRIDE + c);
                float4 x[AD_MAX_CLUSTER];
#pragma unroll
                for (int p = 0; p < AD_MAX_CLUSTER; ++p)
                    if (p < C) x[p] = ld_cluster(at, (u32)p);
#pragma unroll
                for (int p = 0; p < AD_MAX_CLUSTER; ++p)
                    if (p < C) { v[q].x += x[p].x; v[q].y += x[p].y; v[q].z += x[p].z; v[q].w += x[p].w; }
                v[q].x = c < rank ? f * v[q].x : 0.0f;
                v[q].y = c + 1 < rank ? f * v[q].y : 0.0f;
                v[q].z = c + 2 < rank ? f * v[q].z : 0.0f;
                v[q].w = c + 3 < rank ? f * v[q].w : 0.0f;
                if (P.h && split == 0 && r < count && r % C == c_rank) {
                    float *o = P.h + (long long)srow[r] * P.ld_h + c;
                    const float w[4] = {v[q].x, v[q].y, v[q].z, v[q].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (c + e < rank) o[e] = w[e];
                }
                most = fmaxf(fmaxf(fmaxf(most, fabsf(v[q].x)), fmaxf(fabsf(v[q].y), fabsf(v[q].z))), fabsf(v[q].w));
            }
        }
        float inv = 1.0f;
        if (std::is_same<T, __half>::value) {       // binary16 has not fp32's range: a power of two per row
#pragma unroll
            for (int o = TPR / 2; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
            const float p2 = pow2_unit(most);
            inv = pow2_inverse(p2);
            if (sub == 0) sfac[r] = p2;
        }
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            const int c = 4 * (q * TPR + sub);
            if (c < r16) {
                const float x[4] = {v[q].x, v[q].y, v[q].z, v[q].w};
                if constexpr (E == 2) {
                    u16 p[4][PARTS];
#pragma unroll
                    for (int e = 0; e < 4; ++e) split16<T, PARTS>(x[e] * inv, p[e]);
#pragma unroll
                    for (int s = 0; s < PARTS; ++s)
                        *reinterpret_cast<uint2 *>(ho + (s * TM + r) * G::HO_STRIDE + 2 * c) =
                            make_uint2((u32)p[0][s] | ((u32)p[1][s] << 16), (u32)p[2][s] | ((u32)p[3][s] << 16));
                } else {
                    *reinterpret_cast<float4 *>(ho + r * G::HO_STRIDE + 4 * c) = v[q];
                }
            }
        }
    }
    __syncwarp();               // (stores above diverge; the barrier wants whole warps)
    cluster_arrive();           // this CTA has read its peers' sums
    __syncthreads();
    // ---- expand: a lane has U neighbouring columns of each of its two rows
    float row_f[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) row_f[h] = std::is_same<T, __half>::value ? factor * sfac[rg * 16 + g + 8 * h] : factor;
    auto load_h = [&](FragA<T> &a, int s, int p) {
        const char *at = ho + (p * TM + rg * 16 + g) * G::HO_STRIDE + (s * KSTEP + t4 * (KSTEP / 4)) * E;
        frag_h(a, *reinterpret_cast<const uint2 *>(at), *reinterpret_cast<const uint2 *>(at + 8 * G::HO_STRIDE));
    };
    constexpr bool HOLD = RP <= 32 && E == 2;                // h stays in registers
    FragA<T> hold[HOLD ? ST : 1][PARTS];
    if constexpr (HOLD) {
#pragma unroll
        for (int s = 0; s < ST; ++s)
            if (s * KSTEP < r16)
#pragma unroll
                for (int p = 0; p < PARTS; ++p) load_h(hold[s][p], s, p);
    }
    // (fp32, whose result is not rounded to 16 bits: the truncated sums of two steps, 6 products, are added with rounding)
    constexpr int GROUP = E == 4 ? 2 : ST;
    static_assert(SH % 2 == 0 || SH == ST, "whole groups");
    float d[NT][4];
    auto expand = [&](const DstB &x, int s0) {
        float e[NT][4];
#pragma unroll
        for (int s = 0; s < SH; ++s) {
            if (s0 + s && (s0 + s) * KSTEP >= r16) break;
            const bool later = s0 + s >= GROUP, opens = (s0 + s) % GROUP == 0;
            FragB<T> b[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) frag_b(b[j], x.b[s][j].x, x.b[s][j].y);
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p) {
                FragA<T> a;
                if constexpr (HOLD) a = hold[s][p];
                else load_h(a, s0 + s, p);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    if (opens && p == PARTS - 1) mma_first(later ? e[j] : d[j], a, b[j]);
                    else mma_step(later ? e[j] : d[j], a, b[j]);
                }
            }
            if (later && (s0 + s) % GROUP == GROUP - 1) {
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) d[j][q] += e[j][q];
            }
        }
    };
    auto finish = [&](const DstY &y, char *o0, char *o1, int n) {
        if (live[0]) store_unit<V, E>(o0, add_unit<T, NT>(y.y[0], d, 0, row_f[0]), n);
        if (live[1]) store_unit<V, E>(o1, add_unit<T, NT>(y.y[1], d, 1, row_f[1]), n);
    };
    const long long ahead = blocks > 0 ? KW * BLOCK : 0;             // (the loads run ahead of the stores)
    char *o0 = py[0] - ahead, *o1 = py[1] - ahead;
    auto next = [&]() {
        o0 += KW * BLOCK;
        o1 += KW * BLOCK;
    };
    DstB b1;
    if constexpr (G::AHEAD) {
#pragma unroll 1
        for (int i = 0; i < blocks; i += 2) {
            if (i + 1 < blocks) {
                load_y(y1);
                load_b(b1, 0, KB);
            }
            expand(b0, 0);
            finish(y0, o0, o1, U);
            next();
            if (i + 2 < blocks) {
                load_y(y0);
                load_b(b0, 0, KB);
            }
            if (i + 1 < blocks) {
                expand(b1, 0);
                finish(y1, o0, o1, U);
                next();
            }
        }
    } else {
#pragma unroll 1
        for (int i = 0; i < blocks; i += 2) {
            load_b(b1, SH, KB);
            if (i + 1 < blocks) load_y(y1);
            expand(b0, 0);
            if (i + 1 < blocks) load_b(b0, 0, KB);
            expand(b1, SH);
            finish(y0, o0, o1, U);
            next();
            if (i + 1 < blocks) {
                load_b(b1, SH, KB);
                if (i + 2 < blocks) load_y(y0);
                expand(b0, 0);
                if (i + 2 < blocks) load_b(b0, 0, KB);
                expand(b1, SH);
                finish(y1, o0, o1, U);
                next();
            }
        }
    }
    if (nb0 + blocks * KW < nb1) {              // the last block, in part
        const int left = wd - (nb0 + blocks * KW) * KB, n = min(max(left - t4 * U, 0), U);
        y0.y[0] = load_some<E>(o0, n);
        y0.y[1] = load_some<E>(o1, n);
#pragma unroll
        for (int s0 = 0; s0 < ST; s0 += SH) {
            load_b(b0, s0, left - 1);
            expand(b0, s0);
        }
        finish(y0, o0, o1, n);
    }
    __syncwarp();
    cluster_wait();             // peers may still read this CTA's sums until here
}

// ------------------------------------------------------------------ weight gradients
// dA = u^T x and dB = scale * dy^T h: for each adapter, a sum over its rows of a column (u or h, `rank` numbers) times
// a row of activations (x or dy). A CTA takes a strip of activation columns and a share of the adapter's
// rows, 64 at a time; the CTAs that share an adapter's rows are a cluster and add their sums over distributed
// shared memory, in order, so there are neither atomics nor a second launch. The coefficients are fp32 and the
// results too, so they enter the products with their whole precision: three 16-bit parts in bfloat16, two in
// binary16 under a power of two per rank and tile.
struct WgEntry {
    float *out[2];           // dA, dB; NULL: not formed
    float scale;
    int rank;
    int n_rows;
    u16 run0, n_runs;
};
static_assert(sizeof(WgEntry) == 32, "packed into the parameters");

struct WgSide {
    const void *act;         // x | dy
    const float *coef;       // u | h
    long long ld_act, ld_coef, width;
    int vec_act, vec_coef;
};

struct WgradParams {
    WgSide side[2];
    int strips0;             // strips of side 0; the others are side 1's
    int accumulate;
    int n_entries;
    int pad;
    u32 blob[AD_BLOB / 4];   // entries, runs
};
static_assert(sizeof(WgradParams) <= 4096, "kernel parameters");

// What the two kernels below share: a CTA's place, its rows by number, its copies, and the sum over the cluster.
struct WgPlace {
    int sd, rank, r16, n_rows, n_runs, t0, nt, wide;
    long long col0;
    const AdapterRun *runs;
    float *out;
    float scale;
};
__device__ __forceinline__ WgPlace wg_place(const WgradParams &P, int wc)
{
    WgPlace w;
    const int C = (int)cluster_size(), c_rank = (int)cluster_rank();
    const WgEntry *entries = reinterpret_cast<const WgEntry *>(P.blob);
    const WgEntry &ent = entries[blockIdx.y / C];
    w.sd = (int)blockIdx.x >= P.strips0 ? 1 : 0;
    w.runs = reinterpret_cast<const AdapterRun *>(entries + P.n_entries) + ent.run0;
    w.out = ent.out[w.sd];
    w.scale = w.sd ? ent.scale : 1.0f;
    w.rank = ent.rank;
    w.r16 = (ent.rank + 15) & ~15;
    w.n_rows = ent.n_rows;
    w.n_runs = ent.n_runs;
    w.col0 = (long long)((int)blockIdx.x - (w.sd ? P.strips0 : 0)) * wc;
    w.wide = (int)min((long long)wc, P.side[w.sd].width - w.col0);
    const int tiles = (ent.n_rows + AD_WG_ROWS - 1) / AD_WG_ROWS;
    w.t0 = (int)((long long)c_rank * tiles / C);
    w.nt = (int)((long long)(c_rank + 1) * tiles / C) - w.t0;
    return w;
}
// Rows of the CTA's tile i, -1 past the end, into slot i & 7 of `srow`. By threads t, t + 32, ... of a warp, or the first 64.
__device__ __forceinline__ void wg_number_rows(const WgPlace &w, int *srow, int i, int t, int step)
{
    if (i >= w.nt) return;
    if (w.n_runs == 1) {
        for (; t < AD_WG_ROWS; t += step) {
            const int r = (w.t0 + i) * AD_WG_ROWS + t;
            srow[(i & 7) * AD_WG_ROWS + t] = r < w.n_rows ? w.runs[0].first + r : -1;
        }
        return;
    }
    for (; t < AD_WG_ROWS; t += step) {
        const int r = (w.t0 + i) * AD_WG_ROWS + t;
        srow[(i & 7) * AD_WG_ROWS + t] = r < w.n_rows ? adapter_row(w.runs, w.n_runs, r) : -1;
    }
}
// `so` [rank][stride]: this CTA's sums. Each CTA of the cluster adds its share of the columns, in order of the ranks.
__device__ __forceinline__ void wg_finish(const WgradParams &P, const WgPlace &w, float *so, int stride, int wc)
{
    const int C = (int)cluster_size(), c_rank = (int)cluster_rank(), rank = w.rank;
    cluster_arrive();
    cluster_wait();
    const u32 so_u = smem_u32(so);
    const int quads = rank * (wc / 4);
    for (int u = (int)threadIdx.x < THREADS ? c_rank * THREADS + (int)threadIdx.x : quads; u < quads; u += C * THREADS) {
        // dA is written along its rows, dB (whose rows are `rank` numbers) along the ranks
        const int m = w.sd ? u % rank : u / (wc / 4), c = (w.sd ? u / rank : u % (wc / 4)) * 4;
        if (c >= w.wide) continue;
        const u32 at = so_u + (m * stride + c) * 4;
        float4 x[AD_MAX_CLUSTER], v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int p = 0; p < AD_MAX_CLUSTER; ++p)
            if (p < C) x[p] = ld_cluster(at, (u32)p);
#pragma unroll
        for (int p = 0; p < AD_MAX_CLUSTER; ++p)
            if (p < C) { v.x += x[p].x; v.y += x[p].y; v.z += x[p].z; v.w += x[p].w; }
        const float o[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < w.wide) {
                float *to = w.out + (w.sd ? (w.col0 + c + e) * rank + m : (long long)m * P.side[0].width + w.col0 + c + e);
                *to = P.accumulate ? *to + o[e] : o[e];
            }
    }
    if (w.sd) pdl_wait();       // no CTA leaves ahead of the kernel before
    __syncwarp();
    cluster_arrive();
    cluster_wait();             // peers may still read this CTA's sums until here
}

// ---- fp32: TF32 parts on the warp-level instruction, operands from shared memory. (Two parts of 11 bits and fp32's
// exponents hold all but the last two bits of a value; three products of them, the small one by the small one left out.)
template <int RP>
struct WgGeom32 {
    static constexpr int R = AD_WG_ROWS, WC = 128, NTW = WC / 64;      // columns of a strip; 8-column tiles of a warp
    static constexpr int X_STRIDE = WC * 4 + 16, F_STRIDE = RP * 4 + 16;
    static constexpr int STAGE = R * (X_STRIDE + F_STRIDE);
    static constexpr int O_STRIDE = WC + 4;                            // floats: this CTA's sums, [rank][column]
    static constexpr int FIXED = 8 * R * 4;                            // row numbers of eight tiles
    static constexpr int STAGES = FIXED + 2 * STAGE <= 113 * 1024 ? 2 : FIXED + 3 * STAGE <= 227 * 1024 ? 3 : 2;
    static constexpr int SMEM = FIXED + STAGES * STAGE;
    static_assert(SMEM <= 227 * 1024 && STAGE % 16 == 0, "shared memory");
    static_assert(RP * O_STRIDE * 4 <= STAGES * STAGE, "the sums lie where the stages were");
};

template <int RP, int V>
__global__ void __launch_bounds__(THREADS) k_adapter_wgrad32(const __grid_constant__ WgradParams P)
{
    using G = WgGeom32<RP>;
    constexpr int NTW = G::NTW, R = G::R;
    extern __shared__ __align__(128) char sm[];
    int *srow = reinterpret_cast<int *>(sm);
    const u32 ring = smem_u32(sm + G::FIXED);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const WgPlace w = wg_place(P, G::WC);
    if (!w.out) {                                                      // (all CTAs of the cluster leave)
        pdl_wait();
        return;
    }
    const WgSide &S = P.side[w.sd];
    constexpr int XU = G::WC / 4, XN = R * XU / THREADS, FU = RP / 4, FN = R * FU / THREADS;
    const int xq = (tid % XU) * 16, xr = tid / XU, fq = (tid % FU) * 16, fr = tid / FU;
    const int xn = min(max(w.wide * 4 - xq, 0), 16), fn = min(max(w.rank * 4 - fq, 0), 16);
    const char *act = (const char *)S.act, *coef = (const char *)S.coef;
    const char *xbase = act + w.col0 * 4 + xq;
    const long long ldx = S.ld_act * 4, ldf = S.ld_coef * 4;
    const int vec_act = S.vec_act, vec_coef = S.vec_coef;
    auto issue = [&](int i) {
        if (i >= w.nt) return;
        const u32 st = ring + (u32)(i % G::STAGES) * G::STAGE, sf = st + R * G::X_STRIDE;
        const int *rows = srow + (i & 7) * R;
#pragma unroll
        for (int j = 0; j < XN; ++j) {           // (rows that do not exist become zero: they are summed over)
            const int r = xr + THREADS / XU * j, row = rows[r];
            copy_unit<V>(st + r * G::X_STRIDE + xq, xbase + row * ldx, act, row >= 0 ? xn : 0, vec_act);
        }
        if (fq < w.r16 * 4) {
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const int r = fr + THREADS / FU * j, row = rows[r];
                copy_unit<0>(sf + r * G::F_STRIDE + fq, coef + row * ldf + fq, coef, row >= 0 ? fn : 0, vec_coef);
            }
        }
    };
    float acc[RP / 16][NTW][4];
#pragma unroll
    for (int m = 0; m < RP / 16; ++m)
#pragma unroll
        for (int n = 0; n < NTW; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[m][n][q] = 0.0f;
#pragma unroll
    for (int i = 0; i < G::STAGES; ++i) wg_number_rows(w, srow, i, tid, THREADS);
    __syncthreads();
    if (w.sd == 0) pdl_wait();                                         // u is the kernel before's; x, dy and h are not
#pragma unroll 1
    for (int i = 1 - G::STAGES; i < w.nt; ++i) {
        if (i >= 0) {
            cp_wait<G::STAGES - 2>();
            __syncthreads();
        }
        issue(i + G::STAGES - 1);
        cp_commit();
        if (i < 0) continue;
        wg_number_rows(w, srow, i + G::STAGES, tid, THREADS);
        const u32 st = ring + (u32)(i % G::STAGES) * G::STAGE, sf = st + R * G::X_STRIDE;
        // 32 rows at a time, their sums apart from the others: the matrix instruction truncates
        constexpr int HK = 32 / 8;
#pragma unroll 1
        for (int k0 = 0; k0 < R; k0 += 32) {
            FragB<float> b[HK][NTW / 2][2];
#pragma unroll
            for (int k = 0; k < HK; ++k)
#pragma unroll
                for (int n = 0; n < NTW / 2; ++n) load_b2_t(b[k][n], st + (k0 + k * 8) * G::X_STRIDE + (warp * NTW * 8 + n * 16) * 4, G::X_STRIDE, lane);
#pragma unroll
            for (int m = 0; m < RP / 16; ++m) {
                if (m * 16 >= w.r16) break;
                float d[NTW][4];
#pragma unroll
                for (int k = 0; k < HK; ++k) {
                    FragA<float> a;
                    load_a_t(a, sf + (k0 + k * 8) * G::F_STRIDE + m * 64, G::F_STRIDE, lane);
#pragma unroll
                    for (int n = 0; n < NTW; ++n) {
                        if (k == 0) mma_first(d[n], a, b[k][n >> 1][n & 1]);
                        else mma_step(d[n], a, b[k][n >> 1][n & 1]);
                    }
                }
#pragma unroll
                for (int n = 0; n < NTW; ++n)
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[m][n][q] += d[n][q];
            }
        }
    }
    cp_wait<0>();
    __syncthreads();
    float *so = reinterpret_cast<float *>(sm + G::FIXED);
    const int g = lane >> 2, t4 = lane & 3;
#pragma unroll
    for (int m = 0; m < RP / 16; ++m) {
        if (m * 16 >= w.r16) break;
#pragma unroll
        for (int n = 0; n < NTW; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<float2 *>(so + (m * 16 + g + 8 * h) * G::O_STRIDE + warp * NTW * 8 + n * 8 + 2 * t4) =
                    make_float2(w.scale * acc[m][n][2 * h], w.scale * acc[m][n][2 * h + 1]);
    }
    wg_finish(P, w, so, G::O_STRIDE, G::WC);
}

// ---- 16-bit types on tcgen05
// Of 64 rows at a time, the products D[column][rank] = sum over rows of act[row][column] * coef[row][rank] have the rows
// as their depth, and both operands lie in shared memory with the depth as the outer index (MN-major): a strip of 256
// activation columns is two operands A of 128 columns, the coefficients' 16-bit parts are operands B of up to 128
// ranks. Eight warps copy, convert the coefficients and take finished tiles from tensor memory; a ninth issues the
// products of a tile (4 depth steps x 2 operands x 2 or 3 parts, smallest part first). They run while the next tile is
// converted and the tile before is added to fp32 registers, with rounding (the tensor core's own sums are short: 64
// rows). Two accumulators in tensor memory take turns. No warp waits for all others but for the row numbers.
__device__ __forceinline__ void mbar_init(u32 bar, u32 count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory"); }
// Waits for the phase of parity `ph`, at most about a second; false when it did not come.
__device__ __forceinline__ bool mbar_wait(u32 bar, u32 ph)
{
    for (int i = 0; i < (1 << 20); ++i) {
        u32 done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(bar), "r"(ph), "r"(1000u) : "memory");
        if (done) return true;
    }
    return false;
}
template <class T>
__device__ __forceinline__ constexpr u32 umma_idesc(int n)         // fp32 sums; A and B of type T, both MN-major; M = 128
{
    return (1u << 4) | (std::is_same<T, __nv_bfloat16>::value ? (1u << 7) | (1u << 10) : 0u) | (1u << 15) | (1u << 16) | ((u32)(n >> 3) << 17) | (8u << 24);
}
// Shared memory descriptor: start, byte offset of the next group along M or N, of the next eight depth rows, swizzle
// (2: 128 bytes, 4: 64, 6: 32).
__device__ __forceinline__ u64 umma_desc(u32 addr, u32 lbo, u32 sbo, u32 swizzle)
{
    return (u64)((addr & 0x3FFFFu) >> 4) | ((u64)(lbo >> 4) << 16) | ((u64)(sbo >> 4) << 32) | (1ull << 46) | ((u64)swizzle << 61);
}
__device__ __forceinline__ void umma_f16(u32 d, u64 a, u64 b, u32 idesc, u32 add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
// 8 or 16 columns of this warp's lanes of tensor memory; complete only behind tmem_ld_wait().
__device__ __forceinline__ void tmem_ld(u32 addr, float (&v)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "r"(addr));
}
__device__ __forceinline__ void tmem_ld(u32 addr, float (&v)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
                   "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]) : "r"(addr));
}
template <int N, int C>
__device__ __forceinline__ void tmem_ld_wait(float (&v)[N][C])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int s = 0; s < N; ++s)          // (no use of the values may move ahead of the wait)
#pragma unroll
        for (int i = 0; i < C; ++i) asm volatile("" : "+f"(v[s][i]));
}
template <int N> __device__ __forceinline__ void bar_arrive(int id) { asm volatile("bar.arrive %0, %1;" :: "r"(id), "n"(N) : "memory"); }
template <int N> __device__ __forceinline__ void bar_sync(int id) { asm volatile("bar.sync %0, %1;" :: "r"(id), "n"(N) : "memory"); }

// 16-bit parts of two fp32 values, packed; a value that is not finite yields parts that are no numbers.
__device__ __forceinline__ void split_pair(float &x, float &y, u32 &p, __nv_bfloat16)
{
    const __nv_bfloat162 q = __floats2bfloat162_rn(x, y);
    p = *reinterpret_cast<const u32 *>(&q);
    x -= __uint_as_float(p << 16);
    y -= __uint_as_float(p & 0xFFFF0000u);
}
__device__ __forceinline__ void split_pair(float &x, float &y, u32 &p, __half)
{
    const __half2 q = __floats2half2_rn(x, y);
    p = *reinterpret_cast<const u32 *>(&q);
    const float2 f = __half22float2(q);
    x -= f.x;
    y -= f.y;
}

template <class T, int RP>
struct WgGeom16 {
    static constexpr int R = AD_WG_ROWS, WC = 256;                     // rows of a tile, columns of a strip
    static constexpr int PARTS = std::is_same<T, __nv_bfloat16>::value ? 3 : 2;
    static constexpr int STAGE = R * WC * 2;                           // four blocks of 64 columns: [row][128 bytes], swizzled
    // At low ranks the parts lie side by side in one operand (and their sums in tensor memory), so that A is read once
    // for all of them: up to 64 columns of B take the tensor core the same time (53 cycles measured; 68 for 128).
    static constexpr bool SIDE = 4 * PARTS * RP <= 256;
    static constexpr int C_ROW = SIDE || RP >= 64 ? 128 : RP * 2;      // bytes of a row of B (more than 64 ranks: two blocks)
    static constexpr int C_SWIZZLE = SIDE || RP >= 64 ? 2 : RP == 32 ? 4 : 6;
    static constexpr int C_PART = R * RP * 2;
    static constexpr int CONV = SIDE ? R * 128 : PARTS * C_PART;       // one of two
    static constexpr int O_STRIDE = WC + 4;                            // floats: this CTA's sums, [rank][column]
    static constexpr int ROWS = 8 * R * 4;
    // binary16: largest coefficients of a tile by rank (three tiles take turns), and the units that follow from them (two)
    static constexpr int UNITS = std::is_same<T, __half>::value ? (3 + 2) * RP * 4 : 0;
    static constexpr int FIXED = 2 * CONV + ROWS + 128 + UNITS;        // (the swizzled parts first)
    static constexpr int PAD = 1024;                                   // swizzle patterns start at multiples of 1024 bytes
    static constexpr int HALF_SM = 113 * 1024, WHOLE_SM = 227 * 1024;
    static constexpr int stages()
    {
        for (int s = 3; s >= 2; --s)
            if (RP <= 64 && PAD + FIXED + s * STAGE <= HALF_SM) return s;
        for (int s = 4; s >= 2; --s)
            if (PAD + FIXED + s * STAGE <= WHOLE_SM) return s;
        return 2;
    }
    static constexpr int STAGES = stages();
    static constexpr int SMEM = PAD + FIXED + STAGES * STAGE;
    static constexpr int D = SIDE ? PARTS * RP : RP;                   // columns of an accumulator block
    static constexpr int TMEM = 4 * D <= 64 ? 64 : 4 * D <= 128 ? 128 : 4 * D <= 256 ? 256 : 512;    // two accumulators of two blocks
    static constexpr int CTAS = SMEM <= HALF_SM && TMEM <= 256 ? 2 : 1;
    // Two CTAs of 64 ranks are short of registers: ranks are taken from tensor memory 8 at a time, not 16, and the next tile's
    // coefficients are loaded behind that, not ahead of it (2777 rows of ranks 40 to 63: 91 -> 87 us for the call)
    static constexpr bool SHORT = CTAS == 2 && RP == 64;
    static constexpr int TAKE = SHORT ? 8 : 16;
    static constexpr int BLOCK = THREADS + 32;
    static_assert(SMEM <= WHOLE_SM && STAGE % 1024 == 0 && C_PART % 1024 == 0, "shared memory");
    static_assert(STAGES <= 3 || ROWS >= 4 * R * 4, "row numbers of four tiles");
    static_assert(RP * O_STRIDE * 4 <= STAGES * STAGE + 2 * CONV, "the sums lie where the stages and the parts were");
};

// Measured: 8192 rows of 4 adapters, rank 16, 4096 + 4096 columns, bf16: 45 us against 21 us for the bytes; workers
// spend about half of a tile issuing its copies, the rest is the products' latency. 2777 rows of 6 adapters, ranks 40 to
// 63, 1500 + 6000 columns, fp16, copies of 8 bytes: 42 us.
template <class T, int RP, int V>
__global__ void __launch_bounds__(THREADS + 32, WgGeom16<T, RP>::CTAS) k_adapter_wgrad16(const __grid_constant__ WgradParams P)
{
    using G = WgGeom16<T, RP>;
    constexpr int R = G::R, PARTS = G::PARTS;
    constexpr bool HALF = std::is_same<T, __half>::value;
    extern __shared__ char sm_raw[];
    char *sm = sm_raw + ((1024u - (smem_u32(sm_raw) & 1023u)) & 1023u);
    char *stages = sm, *conv = sm + G::STAGES * G::STAGE;              // [2][PARTS][row][C_ROW]
    int *srow = reinterpret_cast<int *>(conv + 2 * G::CONV);           // [8][R]
    u64 *bars = reinterpret_cast<u64 *>(reinterpret_cast<char *>(srow) + G::ROWS);
    u32 *s_tmem = reinterpret_cast<u32 *>(bars + 2);
    u32 *smax = reinterpret_cast<u32 *>(bars + 16);                    // [3][rank], patterns of magnitudes
    float *sunit = reinterpret_cast<float *>(smax + 3 * RP);           // [2][rank]
    const u32 ring = smem_u32(stages), conv_u = smem_u32(conv), bar = smem_u32(bars);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const WgPlace w = wg_place(P, G::WC);
    if (!w.out) {                                                      // (all CTAs of the cluster leave)
        pdl_wait();
        return;
    }
    const WgSide &S = P.side[w.sd];
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(s_tmem)), "r"((u32)G::TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (tid == 0) {
        mbar_init(bar, 1);
        mbar_init(bar + 8, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (HALF && tid < RP) smax[tid] = 0;
#pragma unroll
    for (int i = 0; i <= G::STAGES; ++i) wg_number_rows(w, srow, i, tid, THREADS);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const u32 tmem = *s_tmem;

    // Barriers 1 and 2: a tile is ready to be multiplied (workers arrive, the ninth warp waits); 3 and 4: the row numbers
    // further on are there (the other way round). Each pair takes turns: the side that only arrives may be one tile
    // ahead, never two, since it waits for the other side's barrier (or the products) of the tile between.
    if (warp == WARPS) {                         // ---- the warp that issues the products
        constexpr int GROUPS = G::SIDE ? 1 : PARTS;
        const u32 idesc = umma_idesc<T>(G::SIDE ? PARTS * w.r16 : w.r16);
        const u64 b0 = umma_desc(conv_u, R * 128, 8 * G::C_ROW, G::C_SWIZZLE);
        int stage = 0;
#pragma unroll 1
        for (int i = 0; i < w.nt; ++i) {
            __syncwarp();
            bar_arrive<G::BLOCK>(3 + (i & 1));                         // (the row numbers of tile i + STAGES are there)
            bar_sync<G::BLOCK>(1 + (i & 1));
            if (lane == 0) {
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const u64 a0 = umma_desc(ring + (u32)stage * G::STAGE, R * 128, 1024, 2);
                const u64 bi = b0 + ((u32)(i & 1) * G::CONV >> 4);
                const u32 d = tmem + (u32)(i & 1) * (2 * G::D);
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    if (b * 128 >= w.wide) break;
#pragma unroll
                    for (int s = GROUPS - 1; s >= 0; --s)
#pragma unroll
                        for (int k = 0; k < R / 16; ++k)
                            umma_f16(d + b * G::D, a0 + ((b * (2 * R * 128) + k * 2048) >> 4), bi + ((s * G::C_PART + k * 16 * G::C_ROW) >> 4), idesc,
                                     s < GROUPS - 1 || k > 0);
                }
                asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar + 8 * (i & 1)) : "memory");
            }
            __syncwarp();
            if (++stage == G::STAGES) stage = 0;
            wg_number_rows(w, srow, i + G::STAGES + 1, lane, 32);      // (while they run; nobody reads this slot now)
        }
        __syncthreads();                         // (the workers' last products are in their registers)
        __syncthreads();                         // (their sums are in shared memory)
        wg_finish(P, w, reinterpret_cast<float *>(stages), G::O_STRIDE, G::WC);
        return;
    }

    // ---- the workers
    constexpr int XU = G::WC * 2 / 16, XN = R * XU / THREADS, FU = RP / 4, FN = R * FU / THREADS;
    const int xc = tid % XU, xr = tid / XU, fq = (tid % FU) * 4, fr = tid / FU;          // fq: first of four ranks
    const int xn = min(max(w.wide * 2 - xc * 16, 0), 16);
    const char *act = (const char *)S.act;
    const char *xbase = act + w.col0 * 2 + xc * 16;
    const float *coef = S.coef + fq;
    const long long ldx = S.ld_act * 2, ldf = S.ld_coef;
    const int vec_act = S.vec_act;
    const bool has_f = fq < w.r16, whole_f = fq + 4 <= w.rank, vec_f = S.vec_coef == 16;
    const u32 x_to = (xc >> 3) * (R * 128) + xr * 128 + (((xc & 7) ^ (xr & 7)) << 4);     // (rows of a thread are 8 apart: one swizzle)
    static_assert(THREADS / XU == 8, "rows of a thread");
    auto issue = [&](int i) {                    // activations of tile i
        if (i >= w.nt) return;
        const u32 st = ring + (u32)(i % G::STAGES) * G::STAGE + x_to;
        const int *rows = srow + (i & 7) * R;
        const int first = rows[0], last = rows[R - 1];
        if (last - first == R - 1) {             // 64 rows that follow one another, as most tiles' do
            const char *p = xbase + (first + xr) * ldx;
#pragma unroll
            for (int j = 0; j < XN; ++j) {
                copy_unit<V>(st + j * 1024, p, act, xn, vec_act);
                p += 8 * ldx;
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < XN; ++j) {           // (rows that do not exist become zero: they are summed over)
            const int row = rows[xr + 8 * j];
            copy_unit<V>(st + j * 1024, xbase + row * ldx, act, row >= 0 ? xn : 0, vec_act);
        }
    };
    float4 v[FN];
    auto load_coef = [&](int i) {                // coefficients of tile i
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (i >= w.nt || !has_f) continue;
            const int row = srow[(i & 7) * R + fr + THREADS / FU * j];
            if (row < 0) continue;
            const float *p = coef + row * ldf;
            if (vec_f && whole_f) v[j] = *reinterpret_cast<const float4 *>(p);
            else {
                if (fq < w.rank) v[j].x = p[0];
                if (fq + 1 < w.rank) v[j].y = p[1];
                if (fq + 2 < w.rank) v[j].z = p[2];
                if (fq + 3 < w.rank) v[j].w = p[3];
            }
        }
    };
    // four ranks are 8 bytes: block of 64, 16-byte unit (moved by the swizzle), half of it. (A thread's rows lie a
    // multiple of eight apart: one swizzle)
    static_assert(THREADS / FU % 8 == 0, "rows of a thread");
    u32 c_to[PARTS];
#pragma unroll
    for (int s = 0; s < PARTS; ++s) {
        const int by = (G::SIDE ? s * w.r16 + fq : fq) * 2, un = (by & 127) >> 4;
        const int sw = G::C_ROW == 128 ? un ^ (fr & 7) : G::C_ROW == 64 ? un ^ ((fr >> 1) & 3) : un ^ ((fr >> 2) & 1);
        c_to[s] = (G::SIDE ? 0 : s * G::C_PART) + (by >> 7) * (R * 128) + fr * G::C_ROW + (sw << 4) + (by & 8);
    }
    // this thread's column of the strip, `rank` sums of it
    float acc[RP];
#pragma unroll
    for (int m = 0; m < RP; ++m) acc[m] = 0.0f;
    bool fine = true;
    int which = 0;                               // place of the tile's largest coefficients
    auto collect = [&](int i) {                  // tile i's sums from tensor memory
        const u32 at = tmem + (u32)(i & 1) * (2 * G::D) + (u32)(warp >> 2) * G::D + ((u32)(warp & 3) << 21);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        constexpr int SUMS = G::SIDE ? PARTS : 1, CH = G::TAKE;
#pragma unroll
        for (int q = 0; q < RP; q += CH) {
            if (q && q >= w.r16) break;
            float part[SUMS][CH], t[CH];
#pragma unroll
            for (int s = 0; s < SUMS; ++s) tmem_ld(at + s * w.r16 + q, part[s]);
            tmem_ld_wait(part);
#pragma unroll
            for (int e = 0; e < CH; ++e) {       // the parts' sums, smallest first
                t[e] = part[SUMS - 1][e];
#pragma unroll
                for (int s = SUMS - 2; s >= 0; --s) t[e] += part[s][e];
            }
#pragma unroll
            for (int e = 0; e < CH; e += 4) {
                float *to = acc + q + e;
                if constexpr (HALF) {
                    const float4 u = *reinterpret_cast<const float4 *>(sunit + (i & 1) * RP + q + e);
                    to[0] = fmaf(u.x, t[e], to[0]); to[1] = fmaf(u.y, t[e + 1], to[1]);
                    to[2] = fmaf(u.z, t[e + 2], to[2]); to[3] = fmaf(u.w, t[e + 3], to[3]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) to[j] += t[e + j];
                }
            }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    };
    if (w.sd == 0) pdl_wait();                   // u is the kernel before's; x, dy and h are not
    load_coef(0);
#pragma unroll 1
    for (int i = 0; i < G::STAGES - 1; ++i) {
        issue(i);
        cp_commit();
    }
#pragma unroll 1
    for (int i = 0; i < w.nt; ++i) {
        // binary16 has not fp32's range: each rank's coefficients of a tile are divided by a power of two of their own, so
        // that two parts hold 22 bits of it down to 2^-16 of the largest, however the ranks differ (one is not finite: its
        // rank's sums are not)
        float inv[4] = {1.0f, 1.0f, 1.0f, 1.0f};
        if constexpr (HALF) {
            float most[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const float x[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) most[e] = fmaxf(most[e], fabsf(x[e]));
            }
#pragma unroll
            for (int o = 16; o >= FU; o >>= 1)
#pragma unroll
                for (int e = 0; e < 4; ++e) most[e] = fmaxf(most[e], __shfl_xor_sync(0xFFFFFFFFu, most[e], o));
            u32 *at = smax + which * RP + fq;
            which = which == 2 ? 0 : which + 1;
            if (lane < FU)
#pragma unroll
                for (int e = 0; e < 4; ++e) atomicMax(at + e, __float_as_uint(most[e]));
            __syncwarp();
            bar_sync<THREADS>(5);
            const uint4 all = *reinterpret_cast<const uint4 *>(at);
            most[0] = __uint_as_float(all.x); most[1] = __uint_as_float(all.y); most[2] = __uint_as_float(all.z); most[3] = __uint_as_float(all.w);
            // (the next tile's place: last read ahead of this barrier 5, added to behind the next barrier 3 or 4)
            if (tid < RP) smax[which * RP + tid] = 0;
            float unit[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                unit[e] = pow2_unit(most[e]);
                inv[e] = pow2_inverse(unit[e]);
            }
            // (read behind the next barrier; written again behind the barrier 5 that follows the last reader)
            if (tid < FU) *reinterpret_cast<float4 *>(sunit + (i & 1) * RP + fq) = make_float4(unit[0], unit[1], unit[2], unit[3]);
        }
        char *cv = conv + (i & 1) * G::CONV;
        if (has_f) {
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                float x0 = HALF ? v[j].x * inv[0] : v[j].x, x1 = HALF ? v[j].y * inv[1] : v[j].y;
                float x2 = HALF ? v[j].z * inv[2] : v[j].z, x3 = HALF ? v[j].w * inv[3] : v[j].w;
#pragma unroll
                for (int s = 0; s < PARTS; ++s) {
                    uint2 p;
                    split_pair(x0, x1, p.x, T());
                    split_pair(x2, x3, p.y, T());
                    *reinterpret_cast<uint2 *>(cv + c_to[s] + j * (THREADS / FU) * G::C_ROW) = p;
                }
            }
        }
        cp_wait<G::STAGES - 2>();                                      // this thread's share of tile i is there
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (the tensor core reads it)
        __syncwarp();                                                  // (barriers and tensor memory want whole warps: where lanes went apart they meet first)
        bar_arrive<G::BLOCK>(1 + (i & 1));
        if constexpr (!G::SHORT) load_coef(i + 1);
        // the tile before is complete: its buffers are free for the next copies, its sums can be taken. (A wait that ran out
        // makes the gradients no numbers; nothing more is waited for)
        if (i > 0) fine = fine && mbar_wait(bar + 8 * ((i - 1) & 1), ((i - 1) >> 1) & 1);
        issue(i + G::STAGES - 1);
        cp_commit();
        __syncwarp();
        bar_sync<G::BLOCK>(3 + (i & 1));                               // (the row numbers of tile i + STAGES are there)
        if (i > 0) collect(i - 1);
        if constexpr (G::SHORT) load_coef(i + 1);
    }
    if (w.nt > 0) {
        fine = fine && mbar_wait(bar + 8 * ((w.nt - 1) & 1), ((w.nt - 1) >> 1) & 1);
        __syncwarp();
        collect(w.nt - 1);
    }
    cp_wait<0>();
    __syncthreads();
    // tensor memory goes back before anything waits for another CTA
    if (warp == 0) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"((u32)G::TMEM) : "memory");
    }
    float *so = reinterpret_cast<float *>(stages);
    const int col = (warp >> 2) * 128 + (warp & 3) * 32 + lane;
    const float factor = fine ? w.scale : __uint_as_float(0x7FC00000u);         // a product that never came must not go unseen
#pragma unroll
    for (int m = 0; m < RP; ++m) {
        if (m % 16 == 0 && m && m >= w.r16) break;
        so[m * G::O_STRIDE + col] = factor * acc[m];
    }
    __syncthreads();
    wg_finish(P, w, so, G::O_STRIDE, G::WC);
}

// A and B laid out anew ahead of the row kernel, rows padded with zeros to 16 bytes: for the backward pass transposed (it
// wants B by its columns and A by its columns), for the forward pass where their rows do not allow the accesses that
// it makes (odd ranks, odd widths). They are a small part of what the row kernel moves: 4 to 6 us, most of it the
// launch, where the row kernel on values read one by one lost more (24 against 18 us for 24 adapters in decoding).
struct PackItem {
    const void *src;         // [rows][cols]
    void *dst;               // [rows][ld], or transposed [cols][ld]
    long long rows, cols;
    int ld, trans;
    int block0, pad;         // first CTA of the item
};
constexpr int AD_PACK_MAX = 80, AD_PACK_TILE = 64;
struct PackParams {
    int n, pad;
    PackItem item[AD_PACK_MAX];
};
static_assert(sizeof(PackItem) == 48 && sizeof(PackParams) <= 4096, "kernel parameters");

// A CTA takes a tile of 64 x 64 values through shared memory.
template <class U>
__global__ void __launch_bounds__(THREADS) k_adapter_pack(const __grid_constant__ PackParams P)
{
    __shared__ U t[AD_PACK_TILE][AD_PACK_TILE + 4 / sizeof(U)];
    int which = 0;
    for (int hi = P.n - 1; which < hi;) {
        const int mid = (which + hi + 1) >> 1;
        if (P.item[mid].block0 <= (int)blockIdx.x) which = mid; else hi = mid - 1;
    }
    const PackItem &it = P.item[which];
    const int tile = (int)blockIdx.x - it.block0, across = (int)((it.cols + AD_PACK_TILE - 1) / AD_PACK_TILE);
    const long long r0 = (long long)(tile / across) * AD_PACK_TILE, c0 = (long long)(tile % across) * AD_PACK_TILE;
    const int x = threadIdx.x % AD_PACK_TILE, y = threadIdx.x / AD_PACK_TILE;
    pdl_launch_dependents();
    const int rows = (int)min(it.rows - r0, (long long)AD_PACK_TILE), cols = (int)min(it.cols - c0, (long long)AD_PACK_TILE);
    const U *src = (const U *)it.src + (r0 + y) * it.cols + c0 + x;
    U v[AD_PACK_TILE / 4];
#pragma unroll
    for (int i = 0; i < AD_PACK_TILE / 4; ++i) {
        v[i] = y + 4 * i < rows && x < cols ? *src : U(0);
        src += 4 * it.cols;
    }
#pragma unroll
    for (int i = 0; i < AD_PACK_TILE / 4; ++i) t[y + 4 * i][x] = v[i];
    __syncthreads();
    // rows of the result run along c (as given) or along r (transposed); their padding is written too
    const int o_rows = it.trans ? cols : rows;
    const long long o_row = it.trans ? c0 : r0, o_col = it.trans ? r0 : c0;
    if (o_col + x >= it.ld) return;
    U *dst = (U *)it.dst + (o_row + y) * it.ld + o_col + x;
#pragma unroll
    for (int i = 0; i < AD_PACK_TILE / 4; ++i) {
        const int a = y + 4 * i;
        if (a < o_rows) *dst = it.trans ? t[x][a] : t[a][x];
        dst += 4 * it.ld;
    }
}

}  // namespace cs
