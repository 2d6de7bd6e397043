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
// of the destination columns, whose old values were already on their way. src is read once, dst once
// and written once, h never makes a trip through global memory in between.
//
// The arithmetic is small (2 * rank operations per source and destination element), so the
// kernels are bound by memory up to ranks of 64 or so; the products run on the warp-level matrix instruction
// (operands from shared memory into registers), whose rate is far above what the memory can feed.
// tcgen05 would want 128-row accumulators in tensor memory for an 8- to 64-wide product.
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
constexpr int AD_WG_ROWS = 64;               // rows of a tile of the weight gradients

struct AdapterEntry {                        // an adapter as k_adapter sees it
    const void *shrink;
    const void *expand;
    float scale;
    u16 rank;
    uint8_t vec_s, vec_e;                    // widest access both allow (bytes)
};
static_assert(sizeof(AdapterEntry) == 24, "packed into the parameters");

struct AdapterTile {
    int first;                               // first row, where the rows follow one another
    int list;                                // else: place of their numbers in the row list; -1
    u16 count;
    u16 adapter;                             // place in the parameters
};
static_assert(sizeof(AdapterTile) == 12, "packed into the parameters");

struct AdapterParams {
    const void *src;
    void *dst;                               // NULL: nothing is expanded
    float *h;                                // h (forward) or scale * S src (backward); NULL: not kept
    long long ld_src, ld_dst, ld_h;
    long long width_src, width_dst;
    int vec_src, vec_dst;
    int n_entries, n_tiles;
    u32 blob[AD_BLOB / 4];                   // entries, tiles, rows
};
static_assert(sizeof(AdapterParams) <= 4096, "kernel parameters");

// ------------------------------------------------------------------ types
template <class T> struct AdType {           // 16-bit types
    static constexpr int E = 2, KSTEP = 16, NT = 4;      // bytes; depth of a product step; 8-column tiles of a warp
    static constexpr int PARTS = 2;                      // 16-bit parts of an fp32 operand of the expansion
};
template <> struct AdType<float> {
    static constexpr int E = 4, KSTEP = 8, NT = 2;
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
__device__ __forceinline__ void st_shared2(u32 dst, u16 v) { asm volatile("st.shared.u16 [%0], %1;" :: "r"(dst), "h"(v) : "memory"); }

// 16 bytes of a row into shared memory, the first `left` of them exist (the rest become zero). `vec`: the
// accesses that the row's alignment allows. `any` is some address that may be formed when nothing exists.
__device__ __forceinline__ void copy_unit(u32 dst, const char *src, const char *any, int left, int vec)
{
    left = min(max(left, 0), 16);
    if (vec >= 16) {
        cp16(dst, left ? src : any, left);
    } else if (vec == 8) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int n = min(max(left - 8 * i, 0), 8);
            cp8(dst + 8 * i, n ? src + 8 * i : any, n);
        }
    } else if (vec == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = min(max(left - 4 * i, 0), 4);
            cp4(dst + 4 * i, n ? src + 4 * i : any, n);
        }
    } else {
        u32 w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (left > 2 * i) w[i >> 1] |= (u32) * reinterpret_cast<const u16 *>(src + 2 * i) << (16 * (i & 1));
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
__device__ __forceinline__ u32 to_tf32(float x)
{
    u32 r;
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(x));
    return r;
}

// Operand fragments of one product step (16 x KSTEP times KSTEP x 8).
template <class T> struct FragA { u32 r[4]; };
template <class T> struct FragB { u32 r[2]; };
template <> struct FragA<float> { u32 hi[4], lo[4]; };       // two TF32 parts: 22 bits of the operand
template <> struct FragB<float> { u32 hi[2], lo[2]; };

__device__ __forceinline__ void split_tf32(float x, u32 &hi, u32 &lo)
{
    hi = to_tf32(x);
    const float rest = x - __uint_as_float(hi);
    // an operand that is not finite has no rest
    lo = (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u ? 0u : to_tf32(rest);
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

// A operand from [m][k] at `base` (rows of `stride` bytes).
template <class T>
__device__ __forceinline__ void load_a(FragA<T> &f, u32 base, int stride, int lane)
{
    ldsm4(f.r, base + (lane & 15) * stride + (lane >> 4) * 16);
}
__device__ __forceinline__ void load_a(FragA<float> &f, u32 base, int stride, int lane)
{
    const u32 p = base + (lane >> 2) * stride + (lane & 3) * 4;
    split_tf32(lds_f32(p), f.hi[0], f.lo[0]);
    split_tf32(lds_f32(p + 8 * stride), f.hi[1], f.lo[1]);
    split_tf32(lds_f32(p + 16), f.hi[2], f.lo[2]);
    split_tf32(lds_f32(p + 8 * stride + 16), f.hi[3], f.lo[3]);
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
// B operands of two neighbouring 8-column tiles from [n][k].
template <class T>
__device__ __forceinline__ void load_b2(FragB<T> (&f)[2], u32 base, int stride, int lane)
{
    u32 r[4];
    const int q = lane >> 3;
    ldsm4(r, base + ((q >> 1) * 8 + (lane & 7)) * stride + (q & 1) * 16);
    f[0].r[0] = r[0]; f[0].r[1] = r[1]; f[1].r[0] = r[2]; f[1].r[1] = r[3];
}
__device__ __forceinline__ void load_b2(FragB<float> (&f)[2], u32 base, int stride, int lane)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const u32 p = base + (i * 8 + (lane >> 2)) * stride + (lane & 3) * 4;
        split_tf32(lds_f32(p), f[i].hi[0], f[i].lo[0]);
        split_tf32(lds_f32(p + 16), f[i].hi[1], f[i].lo[1]);
    }
}
// ... and from [k][n].
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

// Power of two whose inverse brings |x| <= most below 2 (1 where there is nothing to scale).
__device__ __forceinline__ float pow2_above(float most)
{
    const u32 e = (__float_as_uint(most) >> 23) & 0xFFu;
    return (e == 0u || e >= 254u) ? (e == 0u ? 1.1754943508222875e-38f : 1.0f) : __uint_as_float(e << 23);
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

// ------------------------------------------------------------------ geometry
// TM rows of a tile: TM / 16 groups of rows, 8 / (TM / 16) warps side by side in each.
template <class T, bool TRANS, int TM, int RP>
struct AdGeom {
    static constexpr int E = AdType<T>::E, NT = AdType<T>::NT;
    static constexpr int RG = TM / 16, KW = WARPS / RG;
    static constexpr int KC = 256 / E;                               // source columns of a chunk
    static constexpr int NWC = 8 * NT;                               // destination columns of a warp
    static constexpr int NC = NWC * KW;                              // ... of a chunk
    static constexpr int X_STRIDE = 256 + 16;                        // row strides in shared memory: eight rows at a
    static constexpr int S_STRIDE = TRANS ? RP * E + 16 : 256 + 16;  // 16-byte step meet all banks
    static constexpr int S_ROWS = TRANS ? KC : RP;
    static constexpr int Y_STRIDE = NC * E + 64;                     // two rows of four 16-byte accesses meet all banks
    static constexpr int E_STRIDE = TRANS ? NC * E + 16 : RP * E + 16;
    static constexpr int E_ROWS = TRANS ? RP : NC;
    static constexpr int STAGE1 = TM * X_STRIDE + S_ROWS * S_STRIDE;
    static constexpr int STAGE2 = TM * Y_STRIDE + E_ROWS * E_STRIDE;
    static constexpr int STAGE = STAGE1 > STAGE2 ? STAGE1 : STAGE2;
    static constexpr int HP_STRIDE = RP + 4;                         // floats
    static constexpr int HP = (KW > 1 ? KW / 2 : 1) * TM * HP_STRIDE * 4;    // partial sums
    static constexpr int HO_STRIDE = E == 2 ? RP * 2 + 16 : RP * 4 + 16;     // operand of the expansion, bytes
    static constexpr int HO = TM * HO_STRIDE * AdType<T>::PARTS;
    static constexpr int FIXED = HP + HO + TM * 8;
    static constexpr int HALF_SM = 113 * 1024, WHOLE_SM = 227 * 1024;
    static constexpr int stages()
    {
        for (int s = 4; s >= 2; --s)
            if (FIXED + s * STAGE <= HALF_SM) return s;
        return FIXED + 3 * STAGE <= WHOLE_SM ? 3 : 2;
    }
    static constexpr int STAGES = stages();
    static constexpr int SMEM = FIXED + STAGES * STAGE;
    static_assert(SMEM <= WHOLE_SM, "shared memory");
    static_assert(STAGE % 16 == 0 && HP % 16 == 0 && HO % 16 == 0, "alignment");
};

// Where column c of a warp's NWC destination columns is put, so that a thread's accumulators
// (columns 2t, 2t+1 of every 8-column tile) are 2 * NT neighbouring columns of the destination.
template <int NT>
__device__ __forceinline__ int place_of(int c)
{
    const int l = c % (8 * NT), t = l / (2 * NT), j = (l % (2 * NT)) >> 1;
    return c - l + j * 8 + 2 * t + (c & 1);
}

template <class T, bool TRANS, int TM, int RP>
__global__ void __launch_bounds__(THREADS) k_adapter(const __grid_constant__ AdapterParams P)
{
    using G = AdGeom<T, TRANS, TM, RP>;
    constexpr int E = G::E, NT = G::NT, KSTEP = AdType<T>::KSTEP, PARTS = AdType<T>::PARTS;
    extern __shared__ __align__(128) char sm[];
    float *hp = reinterpret_cast<float *>(sm);
    char *ho = sm + G::HP;
    int *srow = reinterpret_cast<int *>(ho + G::HO);
    float *sfac = reinterpret_cast<float *>(srow + TM);
    const u32 ring = smem_u32(sm + G::FIXED);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rg = warp / G::KW, kw = warp % G::KW;
    const int C = (int)cluster_size(), c_rank = (int)cluster_rank();

    const AdapterEntry *entries = reinterpret_cast<const AdapterEntry *>(P.blob);
    const AdapterTile *tiles = reinterpret_cast<const AdapterTile *>(P.blob + P.n_entries * (sizeof(AdapterEntry) / 4));
    const int *row_list = reinterpret_cast<const int *>(tiles + P.n_tiles);
    const AdapterTile tile = tiles[blockIdx.x / C];
    const AdapterEntry ent = entries[tile.adapter];
    const int count = tile.count, rank = ent.rank, r16 = (rank + 15) & ~15;
    if (tid < TM) srow[tid] = tid < count ? (tile.list < 0 ? tile.first + tid : row_list[tile.list + tid]) : 0;
    __syncthreads();

    const int KT = (int)((P.width_src + G::KC - 1) / G::KC), NTt = P.dst ? (int)((P.width_dst + G::NC - 1) / G::NC) : 0;
    const int kc0 = (int)((long long)c_rank * KT / C), nk = (int)((long long)(c_rank + 1) * KT / C) - kc0;
    const int nc0 = (int)((long long)c_rank * NTt / C), nn = (int)((long long)(c_rank + 1) * NTt / C) - nc0;
    const char *src = (const char *)P.src, *shrink = (const char *)ent.shrink, *expand = (const char *)ent.expand;

    // chunk i of this CTA's work (source columns first, then destination columns) into a stage of the ring
    auto issue = [&](int i) {
        const u32 st = ring + (u32)(i % G::STAGES) * G::STAGE;
        if (i < nk) {
            const long long col = (long long)(kc0 + i) * G::KC;
            const int left = (int)min((long long)256, (P.width_src - col) * E);       // bytes of the chunk that exist
            for (int u = tid; u < count * 16; u += THREADS) {
                const int r = u >> 4, q = (u & 15) * 16;
                copy_unit(st + r * G::X_STRIDE + q, src + ((long long)srow[r] * P.ld_src + col) * E + q, src, left - q, P.vec_src);
            }
            const u32 ss = st + TM * G::X_STRIDE;
            if (!TRANS) {
                for (int u = tid; u < rank * 16; u += THREADS) {
                    const int r = u >> 4, q = (u & 15) * 16;
                    copy_unit(ss + r * G::S_STRIDE + q, shrink + ((long long)r * P.width_src + col) * E + q, shrink, left - q, ent.vec_s);
                }
            } else {
                const int upr = r16 * E / 16;
                for (int u = tid; u < G::KC * upr; u += THREADS) {
                    const int r = u / upr, q = (u % upr) * 16;
                    const bool there = col + r < P.width_src;
                    copy_unit(ss + r * G::S_STRIDE + q, shrink + (col + r) * rank * E + q, shrink, there ? rank * E - q : 0, ent.vec_s);
                }
            }
        } else if (i < nk + nn) {
            const long long col = (long long)(nc0 + i - nk) * G::NC;
            const int wide = (int)min((long long)G::NC, P.width_dst - col);            // columns of the chunk that exist
            constexpr int YU = G::NC * E / 16;
            const char *dst = (const char *)P.dst;
            for (int u = tid; u < count * YU; u += THREADS) {
                const int r = u / YU, q = (u % YU) * 16;
                copy_unit(st + r * G::Y_STRIDE + q, dst + ((long long)srow[r] * P.ld_dst + col) * E + q, dst, wide * E - q, P.vec_dst);
            }
            const u32 se = st + TM * G::Y_STRIDE;
            if (!TRANS) {
                const int upr = r16 * E / 16;
                for (int u = tid; u < wide * upr; u += THREADS) {
                    const int c = u / upr, q = (u % upr) * 16;
                    copy_unit(se + place_of<NT>(c) * G::E_STRIDE + q, expand + (col + c) * rank * E + q, expand, rank * E - q, ent.vec_e);
                }
            } else {
                // a 16-byte unit is one thread's columns: its pairs go to NT tiles
                for (int u = tid; u < r16 * YU; u += THREADS) {
                    const int r = u / YU, c = (u % YU) * (16 / E);
                    const char *s = expand + ((long long)r * P.width_dst + col + c) * E;
                    const u32 d = se + r * G::E_STRIDE + place_of<NT>(c) * E;
                    const int left = r < rank ? (wide - c) * E : 0;
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        const int n = min(max(left - 2 * E * j, 0), 2 * E);
                        if (E == 2) {
                            if (ent.vec_e >= 4) cp4(d + j * 16, n ? s + 4 * j : expand, n);
                            else
                                for (int e = 0; e < 2; ++e) st_shared2(d + j * 16 + 2 * e, n > 2 * e ? *reinterpret_cast<const u16 *>(s + 4 * j + 2 * e) : (u16)0);
                        } else {
                            if (ent.vec_e >= 8) cp8(d + j * 32, n ? s + 8 * j : expand, n);
                            else
                                for (int e = 0; e < 2; ++e) cp4(d + j * 32 + 4 * e, n > 4 * e ? s + 8 * j + 4 * e : expand, n > 4 * e ? 4 : 0);
                        }
                    }
                }
            }
        }
    };

    const int total = nk + nn;
#pragma unroll
    for (int i = 0; i < G::STAGES - 1; ++i) {
        issue(i);
        cp_commit();
    }
    // ---- shrink: this CTA's partial h
    float acc[RP / 8][4];
#pragma unroll
    for (int j = 0; j < RP / 8; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[j][q] = 0.0f;
    int i = 0;
    for (; i < nk; ++i) {
        cp_wait<G::STAGES - 2>();
        __syncthreads();
        issue(i + G::STAGES - 1);
        cp_commit();
        const u32 st = ring + (u32)(i % G::STAGES) * G::STAGE, ss = st + TM * G::X_STRIDE;
        constexpr int KPW = G::KC / G::KW;                   // source columns of a warp
#pragma unroll
        for (int k = 0; k < KPW; k += KSTEP) {
            const int kk = kw * KPW + k;
            FragA<T> a;
            load_a(a, st + rg * 16 * G::X_STRIDE + kk * E, G::X_STRIDE, lane);
#pragma unroll
            for (int j = 0; j < RP / 8; j += 2) {
                if (j * 8 >= r16) break;
                FragB<T> b[2];
                if (!TRANS) load_b2(b, ss + j * 8 * G::S_STRIDE + kk * E, G::S_STRIDE, lane);
                else load_b2_t(b, ss + kk * G::S_STRIDE + j * 8 * E, G::S_STRIDE, lane);
                mma_step(acc[j], a, b[0]);
                mma_step(acc[j + 1], a, b[1]);
            }
        }
    }
    // ---- the warps of a row group add up, the upper half handing its sums to the lower
    const int g = lane >> 2, t4 = lane & 3;
    auto spot = [&](int slot, int j, int half) { return hp + ((slot * TM + rg * 16 + g + 8 * half) * G::HP_STRIDE + j * 8 + 2 * t4); };
#pragma unroll
    for (int w = G::KW / 2; w >= 1; w >>= 1) {
        if (kw >= w && kw < 2 * w) {
#pragma unroll
            for (int j = 0; j < RP / 8; ++j) {
                if (j * 8 >= r16) break;
                *reinterpret_cast<float2 *>(spot(kw - w, j, 0)) = make_float2(acc[j][0], acc[j][1]);
                *reinterpret_cast<float2 *>(spot(kw - w, j, 1)) = make_float2(acc[j][2], acc[j][3]);
            }
        }
        __syncthreads();
        if (kw < w) {
#pragma unroll
            for (int j = 0; j < RP / 8; ++j) {
                if (j * 8 >= r16) break;
                const float2 p = *reinterpret_cast<const float2 *>(spot(kw, j, 0)), q = *reinterpret_cast<const float2 *>(spot(kw, j, 1));
                acc[j][0] += p.x; acc[j][1] += p.y; acc[j][2] += q.x; acc[j][3] += q.y;
            }
        }
        __syncthreads();
    }
    if (kw == 0) {
#pragma unroll
        for (int j = 0; j < RP / 8; ++j) {
            if (j * 8 >= r16) break;
            *reinterpret_cast<float2 *>(spot(0, j, 0)) = make_float2(acc[j][0], acc[j][1]);
            *reinterpret_cast<float2 *>(spot(0, j, 1)) = make_float2(acc[j][2], acc[j][3]);
        }
    }
    // ---- the CTAs of the cluster add up, in order of their rank; every one of them needs all of h
    cluster_arrive();
    cluster_wait();
    {
        constexpr int TPR = THREADS / TM;                    // threads of a row
        constexpr int QT = (RP / 4 + TPR - 1) / TPR;         // quads of a thread
        const int r = tid / TPR, sub = tid % TPR;
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
                const float f = TRANS ? ent.scale : 1.0f;
                // rows and columns that do not exist hold what shared memory held before
                v[q].x = r < count && c < rank ? f * v[q].x : 0.0f;
                v[q].y = r < count && c + 1 < rank ? f * v[q].y : 0.0f;
                v[q].z = r < count && c + 2 < rank ? f * v[q].z : 0.0f;
                v[q].w = r < count && c + 3 < rank ? f * v[q].w : 0.0f;
                if (P.h && r < count && r % C == c_rank) {
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
            const float f = pow2_above(most);
            inv = pow2_inverse(f);
            if (sub == 0) sfac[r] = f;
        }
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            const int c = 4 * (q * TPR + sub);
            if (c < r16) {
                const float x[4] = {v[q].x, v[q].y, v[q].z, v[q].w};
                if constexpr (sizeof(T) == 2) {
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
    cluster_arrive();           // this CTA has read its peers' sums
    __syncthreads();
    // ---- expand
    const u32 hob = smem_u32(ho);
    const float factor = TRANS ? 1.0f : ent.scale;
    float row_f[2] = {factor, factor};
    if (std::is_same<T, __half>::value) {
        row_f[0] *= sfac[rg * 16 + g];
        row_f[1] *= sfac[rg * 16 + g + 8];
    }
    for (; i < total; ++i) {
        cp_wait<G::STAGES - 2>();
        __syncthreads();
        issue(i + G::STAGES - 1);
        cp_commit();
        const u32 st = ring + (u32)(i % G::STAGES) * G::STAGE, se = st + TM * G::Y_STRIDE;
        float d[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) d[j][q] = 0.0f;
#pragma unroll
        for (int k = 0; k < RP; k += KSTEP) {
            if (k >= r16) break;
            FragA<T> a[PARTS];
#pragma unroll
            for (int s = 0; s < PARTS; ++s) load_a(a[s], hob + (s * TM + rg * 16) * G::HO_STRIDE + k * E, G::HO_STRIDE, lane);
#pragma unroll
            for (int j = 0; j < NT; j += 2) {
                FragB<T> b[2];
                if (!TRANS) load_b2(b, se + (kw * G::NWC + j * 8) * G::E_STRIDE + k * E, G::E_STRIDE, lane);
                else load_b2_t(b, se + k * G::E_STRIDE + (kw * G::NWC + j * 8) * E, G::E_STRIDE, lane);
#pragma unroll
                for (int s = PARTS - 1; s >= 0; --s) {
                    mma_step(d[j], a[s], b[0]);
                    mma_step(d[j + 1], a[s], b[1]);
                }
            }
        }
        // this thread's 2 * NT neighbouring columns of two rows
        const int cl = kw * G::NWC + t4 * 2 * NT;
        const long long col = (long long)(nc0 + i - nk) * G::NC + cl;
        const int wide = (int)min((long long)(2 * NT), P.width_dst - col);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int r = rg * 16 + g + 8 * half;
            if (r >= count || wide <= 0) continue;
            const uint4 old = *reinterpret_cast<const uint4 *>(sm + G::FIXED + (i % G::STAGES) * G::STAGE + r * G::Y_STRIDE + cl * E);
            const u32 o[4] = {old.x, old.y, old.z, old.w};
            u32 w[4];
            if constexpr (E == 2) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    T lo, hi;
                    *reinterpret_cast<u16 *>(&lo) = (u16)(o[j] & 0xFFFF);
                    *reinterpret_cast<u16 *>(&hi) = (u16)(o[j] >> 16);
                    const T x = (T)((float)lo + row_f[half] * d[j][2 * half]), y = (T)((float)hi + row_f[half] * d[j][2 * half + 1]);
                    w[j] = (u32) * reinterpret_cast<const u16 *>(&x) | ((u32) * reinterpret_cast<const u16 *>(&y) << 16);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = __float_as_uint(__uint_as_float(o[j]) + row_f[half] * d[j >> 1][2 * half + (j & 1)]);
            }
            char *out = (char *)P.dst + ((long long)srow[r] * P.ld_dst + col) * E;
            if (wide == 2 * NT && P.vec_dst >= 16) *reinterpret_cast<uint4 *>(out) = make_uint4(w[0], w[1], w[2], w[3]);
            else if (wide == 2 * NT && P.vec_dst == 8) {
                reinterpret_cast<uint2 *>(out)[0] = make_uint2(w[0], w[1]);
                reinterpret_cast<uint2 *>(out)[1] = make_uint2(w[2], w[3]);
            } else if (E == 4) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < wide) reinterpret_cast<u32 *>(out)[j] = w[j];
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (P.vec_dst == 4 && 2 * j + 1 < wide) reinterpret_cast<u32 *>(out)[j] = w[j];
                    else {
                        if (2 * j < wide) reinterpret_cast<u16 *>(out)[2 * j] = (u16)w[j];
                        if (2 * j + 1 < wide) reinterpret_cast<u16 *>(out)[2 * j + 1] = (u16)(w[j] >> 16);
                    }
                }
            }
        }
        __syncwarp();
    }
    cp_wait<0>();
    __syncwarp();
    cluster_wait();             // peers may still read this CTA's sums until here
}

// ------------------------------------------------------------------ weight gradients
// dA = u^T x and dB = scale * dy^T h: for each adapter, a sum over its rows of a column (u or h, `rank` numbers) times
// a row of activations (x or dy). A CTA takes a strip of activation columns and a share of the adapter's
// rows (a split), tile by tile; its sums go to the gradient itself where there is one split, else to the
// workspace, and k_adapter_reduce adds the splits in order. The coefficients are fp32 and the results too,
// so they enter the products with their whole precision: three 16-bit parts in bfloat16, two in binary16 under a
// power of two that follows the largest seen so far.
struct WgEntry {
    float *out[2];           // dA, dB; NULL: not formed
    float scale;
    int rank;
};
struct WgSplit {
    long long slot;          // place of its sums in the workspace (floats); -1: straight into the gradient
    int tile0;
    u16 n_tiles;
    u16 adapter;
};
static_assert(sizeof(WgEntry) == 24 && sizeof(WgSplit) == 16, "packed into the parameters");

struct WgSide {
    const void *act;         // x | dy
    const float *coef;       // u | h
    long long ld_act, ld_coef, width;
    int vec_act, vec_coef;
};

struct WgradParams {
    WgSide side[2];
    float *part;
    int strips0;             // strips of side 0; the others are side 1's
    int accumulate;
    int n_entries, n_splits, n_tiles;
    int pad;
    u32 blob[AD_BLOB / 4];   // entries, splits, tiles, rows
};
static_assert(sizeof(WgradParams) <= 4096, "kernel parameters");

template <class T, int RP>
struct WgGeom {
    static constexpr int E = AdType<T>::E;
    static constexpr int WC = (E == 2 && RP <= 64) ? 256 : 128;        // columns of a strip
    static constexpr int NTW = WC / 64;                                // 8-column tiles of a warp
    static constexpr int X_STRIDE = WC * E + 16, F_STRIDE = RP * 4 + 16, C_STRIDE = RP * 2 + 16;
    static constexpr int PARTS = std::is_same<T, __nv_bfloat16>::value ? 3 : std::is_same<T, __half>::value ? 2 : 0;
    static constexpr int STAGE = AD_WG_ROWS * (X_STRIDE + F_STRIDE);
    static constexpr int CONV = PARTS * AD_WG_ROWS * C_STRIDE;
    static constexpr int FIXED = CONV + 64;
    static constexpr int STAGES = FIXED + 3 * STAGE <= 113 * 1024 ? 3 : FIXED + 2 * STAGE <= 113 * 1024 ? 2 : FIXED + 3 * STAGE <= 227 * 1024 ? 3 : 2;
    static constexpr int SMEM = FIXED + STAGES * STAGE;
    static_assert(SMEM <= 227 * 1024 && STAGE % 16 == 0 && CONV % 16 == 0, "shared memory");
};

template <class T, int RP>
__global__ void __launch_bounds__(THREADS) k_adapter_wgrad(const __grid_constant__ WgradParams P)
{
    using G = WgGeom<T, RP>;
    constexpr int E = G::E, KSTEP = AdType<T>::KSTEP, NTW = G::NTW, R = AD_WG_ROWS;
    constexpr bool HALF = std::is_same<T, __half>::value;
    extern __shared__ __align__(128) char sm[];
    float *smax = reinterpret_cast<float *>(sm + G::CONV);
    const u32 ring = smem_u32(sm + G::FIXED), conv = smem_u32(sm);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int sd = (int)blockIdx.x >= P.strips0 ? 1 : 0;
    const WgSide &S = P.side[sd];
    const WgEntry *entries = reinterpret_cast<const WgEntry *>(P.blob);
    const WgSplit *splits = reinterpret_cast<const WgSplit *>(entries + P.n_entries);
    const AdapterTile *tiles = reinterpret_cast<const AdapterTile *>(splits + P.n_splits);
    const int *row_list = reinterpret_cast<const int *>(tiles + P.n_tiles);
    const WgSplit sp = splits[blockIdx.y];
    const WgEntry ent = entries[sp.adapter];
    float *out = ent.out[sd];
    if (!out) return;
    const int rank = ent.rank, r16 = (rank + 15) & ~15;
    const long long col0 = (long long)((int)blockIdx.x - (sd ? P.strips0 : 0)) * G::WC;
    const int wide = (int)min((long long)G::WC, S.width - col0);

    auto issue = [&](int i) {
        if (i >= sp.n_tiles) return;
        const AdapterTile tile = tiles[sp.tile0 + i];
        const u32 st = ring + (u32)(i % G::STAGES) * G::STAGE;
        auto row_of = [&](int r) { return (long long)(r < tile.count ? (tile.list < 0 ? tile.first + r : row_list[tile.list + r]) : 0); };
        constexpr int XU = G::WC * E / 16;
        for (int u = tid; u < R * XU; u += THREADS) {        // (rows that do not exist become zero: they are summed over)
            const int r = u / XU, q = (u % XU) * 16;
            copy_unit(st + r * G::X_STRIDE + q, (const char *)S.act + (row_of(r) * S.ld_act + col0) * E + q, (const char *)S.act,
                      r < tile.count ? wide * E - q : 0, S.vec_act);
        }
        const u32 sf = st + R * G::X_STRIDE;
        const int upr = r16 / 4;
        for (int u = tid; u < R * upr; u += THREADS) {
            const int r = u / upr, q = (u % upr) * 16;
            copy_unit(sf + r * G::F_STRIDE + q, (const char *)(S.coef + row_of(r) * S.ld_coef) + q, (const char *)S.coef,
                      r < tile.count ? rank * 4 - q : 0, S.vec_coef);
        }
    };

    float acc[RP / 16][NTW][4];
#pragma unroll
    for (int m = 0; m < RP / 16; ++m)
#pragma unroll
        for (int n = 0; n < NTW; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[m][n][q] = 0.0f;
    float top = 0.0f, unit = 1.1754943508222875e-38f;        // binary16: largest coefficient so far, the power of two that goes with it
#pragma unroll
    for (int i = 0; i < G::STAGES - 1; ++i) {
        issue(i);
        cp_commit();
    }
    for (int i = 0; i < sp.n_tiles; ++i) {
        cp_wait<G::STAGES - 2>();
        __syncthreads();
        issue(i + G::STAGES - 1);
        cp_commit();
        const u32 st = ring + (u32)(i % G::STAGES) * G::STAGE;
        const char *sf = sm + G::FIXED + (i % G::STAGES) * G::STAGE + R * G::X_STRIDE;
        if constexpr (E == 2) {
            const int upr = r16 / 4;
            float inv = 1.0f;
            if constexpr (HALF) {
                float most = 0.0f;
                for (int u = tid; u < R * upr; u += THREADS) {
                    const float4 v = *reinterpret_cast<const float4 *>(sf + (u / upr) * G::F_STRIDE + (u % upr) * 16);
                    most = fmaxf(most, fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), fmaxf(fabsf(v.z), fabsf(v.w))));
                }
#pragma unroll
                for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
                if (lane == 0) smax[warp] = most;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < WARPS; ++w) most = fmaxf(most, smax[w]);
                if (most > top) {
                    top = most;
                    const float next = pow2_above(top), shrink = unit * pow2_inverse(next);      // at most 1
                    unit = next;
#pragma unroll
                    for (int m = 0; m < RP / 16; ++m)
#pragma unroll
                        for (int n = 0; n < NTW; ++n)
#pragma unroll
                            for (int q = 0; q < 4; ++q) acc[m][n][q] *= shrink;
                }
                inv = pow2_inverse(unit);
            }
            for (int u = tid; u < R * upr; u += THREADS) {
                const int r = u / upr, c = (u % upr) * 4;
                const float4 v = *reinterpret_cast<const float4 *>(sf + r * G::F_STRIDE + c * 4);
                const float x[4] = {v.x, v.y, v.z, v.w};
                u16 p[4][G::PARTS];
#pragma unroll
                for (int e = 0; e < 4; ++e) split16<T, G::PARTS>(HALF ? x[e] * inv : x[e], p[e]);
#pragma unroll
                for (int s = 0; s < G::PARTS; ++s)
                    *reinterpret_cast<uint2 *>(sm + (s * R + r) * G::C_STRIDE + 2 * c) =
                        make_uint2((u32)p[0][s] | ((u32)p[1][s] << 16), (u32)p[2][s] | ((u32)p[3][s] << 16));
            }
            __syncthreads();
        }
#pragma unroll 1
        for (int k = 0; k < R; k += KSTEP) {
            FragB<T> b[NTW / 2][2];
#pragma unroll
            for (int n = 0; n < NTW / 2; ++n) load_b2_t(b[n], st + k * G::X_STRIDE + (warp * NTW * 8 + n * 16) * E, G::X_STRIDE, lane);
#pragma unroll
            for (int m = 0; m < RP / 16; ++m) {
                if (m * 16 >= r16) break;
                if constexpr (E == 2) {
#pragma unroll
                    for (int s = G::PARTS - 1; s >= 0; --s) {
                        FragA<T> a;
                        load_a_t(a, conv + (s * R + k) * G::C_STRIDE + m * 32, G::C_STRIDE, lane);
#pragma unroll
                        for (int n = 0; n < NTW; ++n) mma_step(acc[m][n], a, b[n >> 1][n & 1]);
                    }
                } else {
                    FragA<T> a;
                    load_a_t(a, smem_u32(sf) + k * G::F_STRIDE + m * 64, G::F_STRIDE, lane);
#pragma unroll
                    for (int n = 0; n < NTW; ++n) mma_step(acc[m][n], a, b[n >> 1][n & 1]);
                }
            }
        }
    }
    cp_wait<0>();
    const float factor = (sd ? ent.scale : 1.0f) * (HALF ? unit : 1.0f);
    const bool direct = sp.slot < 0, add = direct && P.accumulate;
    float *o = direct ? out : P.part + sp.slot + (sd ? (long long)rank * P.side[0].width : 0);
    const int g = lane >> 2, t4 = lane & 3;
#pragma unroll
    for (int m = 0; m < RP / 16; ++m)
#pragma unroll
        for (int n = 0; n < NTW; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int row = m * 16 + g + (q >> 1) * 8, c = warp * NTW * 8 + n * 8 + 2 * t4 + (q & 1);
                if (row < rank && c < wide) {
                    float *to = o + (sd ? (col0 + c) * rank + row : (long long)row * S.width + col0 + c);
                    const float v = factor * acc[m][n][q];
                    *to = add ? *to + v : v;
                }
            }
}

// Adds the splits of each gradient, in order; an adapter without rows gets zeros.
struct RedEntry {
    float *out[2];
    long long slot;          // first split's sums
    int splits;
    int rank;
};
constexpr int AD_RED_MAX = 120;
struct ReduceParams {
    const float *part;
    long long width[2];
    int accumulate;
    int pad;
    RedEntry e[AD_RED_MAX];
};
static_assert(sizeof(ReduceParams) <= 4096, "kernel parameters");

__global__ void __launch_bounds__(THREADS) k_adapter_reduce(const __grid_constant__ ReduceParams P)
{
    const RedEntry &r = P.e[blockIdx.y];
    const long long n0 = (long long)r.rank * P.width[0], n = n0 + (long long)r.rank * P.width[1];
    for (long long i = (long long)blockIdx.x * THREADS + threadIdx.x; i < n; i += (long long)gridDim.x * THREADS) {
        float *out = r.out[i < n0 ? 0 : 1];
        if (!out) continue;
        float *to = out + (i < n0 ? i : i - n0);
        const float *p = P.part + r.slot + i;
        float sum = 0.0f;
#pragma unroll 4
        for (int s = 0; s < r.splits; ++s) sum += __ldcg(p + s * n);
        *to = P.accumulate ? *to + sum : sum;
    }
}

}  // namespace cs
