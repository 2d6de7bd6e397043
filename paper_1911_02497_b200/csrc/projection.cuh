// Products with a projection held in 8 bits: D[output column][row] = sum over the depth of weight * row, on the tensor
// cores' block-scaled form (tcgen05.mma kind::mxf8f6f4): E4M3 codes from shared memory, scale bytes from tensor memory,
// fp32 sums in tensor memory. Scales being powers of two, the instruction applies them exactly, and nothing has to leave
// tensor memory between two groups of the depth.
//
// The weights are operand A, 128 output columns at a time, so that a few rows (a decoding step) are a narrow operand B and
// cost no more of the tensor core than they are. Forward the depth is k, and a tile of weights lies as in memory, depth
// innermost (K-major); backward the depth is n, and the same 128 x 128 box of the same codes is read the other way round
// (MN-major). An instruction takes 32 of the depth; the four of a group of 128 use the same scale byte, chosen by the
// instruction descriptor among the four bytes of a tensor memory word, which therefore holds four groups (a quad).
#pragma once
#include <cuda.h>

#include "coded.cuh"

namespace cs {

constexpr int PJ_WIDE = 128;            // output columns of a tile
constexpr int PJ_QUAD = 4;              // groups of the depth whose scales share a word
constexpr int PJ_STAGES = 12;           // most stages of the ring
constexpr int PJ_SLOTS = 4;             // quads of scales in shared memory
constexpr int PJ_A = GROUP * PJ_WIDE;   // bytes of a stage's weights
constexpr int PJ_SCALES = 1024;         // bytes of a quad's scales: weights, rows
constexpr int PJ_PAD = 1024;            // swizzle patterns start at multiples of 1024 bytes
constexpr int PJ_MAX_TILE = 128;        // rows of a tile

struct ProjectionParams {
    CUtensorMap w, x;                   // codes, boxes of 128 bytes x 128 resp. `tile` rows
    const u8 *w_scales, *x_scales;
    long long w_depth, w_wide;          // distance of the weights' scales by group of the depth, by 128 output columns
    long long ld_xs, ldo;
    void *out;
    long long rows;
    int width, groups;                  // output columns, groups of the depth
    int blocks;                         // of 128 output columns
    int tile;                           // rows of a tile, a multiple of 16
    int stages, ring;                   // ring: bytes of the stages, or of the sums that lie there in the end
    int access;                         // values of a row of the result that may be written at once
    u32 columns;                        // of tensor memory
};

__device__ __forceinline__ u32 smem_u32(const void *p) { return (u32)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(u32 bar, u32 count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void mbar_expect(u32 bar, u32 bytes) { asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory"); }
__device__ __forceinline__ void mbar_arrive(u32 bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory"); }
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
// A box of a tensor map, from column x (a multiple of 128) and row y.
__device__ __forceinline__ void tma_load(u32 dst, const CUtensorMap *map, int x, int y, u32 bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// Shared memory descriptor: start, byte offset of the next eight rows; swizzle 2: 128 bytes, 0: none.
__device__ __forceinline__ u64 umma_desc(u32 addr, u32 sbo, u32 swizzle)
{
    return (u64)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((u64)(sbo >> 4) << 32) | (1ull << 46) | ((u64)swizzle << 61);
}
// Instruction descriptor: E4M3 x E4M3, scales of 8 exponent bits, A MN-major or not, m x n.
__device__ __forceinline__ u32 umma_idesc(bool a_mn, int m, int n) { return (a_mn ? 1u << 15 : 0u) | ((u32)(n >> 3) << 17) | (1u << 23) | ((u32)(m >> 4) << 24); }
// ... with the byte of the scale words that this instruction uses
__device__ __forceinline__ u32 umma_idesc_at(u32 idesc, u32 byte) { return idesc | byte << 29 | byte << 4; }
__device__ __forceinline__ void umma_scaled(u32 d, u64 a, u64 b, u32 idesc, u32 scale_a, u32 scale_b, u32 add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\ttcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(scale_a), "r"(scale_b), "r"(add) : "memory");
}
// 512 bytes of scales, 32 lanes of four words, into four columns of tensor memory (all four groups of 32 lanes).
__device__ __forceinline__ void scales_to_tmem(u32 tmem, u64 desc)
{
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" :: "r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void umma_commit(u32 bar) { asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory"); }
// 16 columns of this warp's lanes; complete only behind tmem_ld_wait().
__device__ __forceinline__ void tmem_ld(u32 addr, float (&v)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
                   "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]) : "r"(addr));
}
__device__ __forceinline__ void tmem_ld_wait(float (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) asm volatile("" : "+f"(v[i]));          // (no use of the values may move ahead of the wait)
}

// The scale bytes of a quad: of 128 output columns' weights, the same for all of them ...
__device__ __forceinline__ u32 weight_scales(const ProjectionParams &P, int quad, long long block)
{
    u32 word = 0;
#pragma unroll
    for (int b = 0; b < PJ_QUAD; ++b) {
        const int g = quad * PJ_QUAD + b;
        if (g < P.groups) word |= (u32)P.w_scales[g * P.w_depth + block * P.w_wide] << (8 * b);
    }
    return word;
}
// ... and of a row (past the last one: anything, its sums are not used).
__device__ __forceinline__ u32 row_scales(const ProjectionParams &P, int quad, long long row)
{
    if (row >= P.rows) return 0;
    const u8 *s = P.x_scales + row * P.ld_xs + quad * PJ_QUAD;
    if (quad * PJ_QUAD + PJ_QUAD <= P.groups) return *reinterpret_cast<const u32 *>(s);
    u32 word = 0;
#pragma unroll
    for (int b = 0; b < PJ_QUAD - 1; ++b)
        if (quad * PJ_QUAD + b < P.groups) word |= (u32)s[b] << (8 * b);
    return word;
}

// A cluster of CTAs takes a tile: its CTAs share the depth by quads, each leaves its sums in its own shared memory, and
// each adds up a part of the tile's rows over all of them, in their order, by distributed shared memory.
// Four warps: copies, products, scales, tensor memory; then all take the sums.
template <class T, bool TRANS>
__global__ void __launch_bounds__(128) k_projection(const __grid_constant__ ProjectionParams P)
{
    extern __shared__ char pj_raw[];
    __shared__ u64 bars[2 * PJ_STAGES + 2 * PJ_SLOTS + 1];
    __shared__ u32 s_tmem;
    __shared__ int s_fail;
    char *ring = pj_raw + ((PJ_PAD - (smem_u32(pj_raw) & (PJ_PAD - 1))) & (PJ_PAD - 1));
    char *scales = ring + P.ring;
    const u32 ring_u = smem_u32(ring), scales_u = smem_u32(scales);
    const u32 full = smem_u32(bars), empty = full + 8 * PJ_STAGES, sc_full = empty + 8 * PJ_STAGES, sc_empty = sc_full + 8 * PJ_SLOTS,
              done = sc_empty + 8 * PJ_SLOTS;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
    const u32 where = blockIdx.x / (u32)parts;
    const int block = (int)(where % (u32)P.blocks);
    const long long row0 = (long long)(where / (u32)P.blocks) * P.tile;
    const int quads = (P.groups + PJ_QUAD - 1) / PJ_QUAD, q0 = (int)((long long)quads * part / parts), q1 = (int)((long long)quads * (part + 1) / parts);
    const int g0 = q0 * PJ_QUAD, g1 = min(q1 * PJ_QUAD, P.groups);
    const int stage_bytes = PJ_A + P.tile * GROUP;

    if (tid == 0) {
        asm volatile("prefetch.tensormap [%0];" :: "l"(&P.w) : "memory");
        asm volatile("prefetch.tensormap [%0];" :: "l"(&P.x) : "memory");
        for (int s = 0; s < PJ_STAGES; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < PJ_SLOTS; ++s) {
            mbar_init(sc_full + 8 * s, 1);
            mbar_init(sc_empty + 8 * s, 1);
        }
        mbar_init(done, 1);
        s_fail = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 3) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&s_tmem)), "r"(P.columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const u32 tmem = s_tmem;
    pdl_wait();
    pdl_launch_dependents();

    if (warp == 0) {                    // ---- copies
        if (lane == 0) {
            int stage = 0;
            u32 turn = 0;
            for (int g = g0; g < g1; ++g) {
                if (g - g0 >= P.stages && !mbar_wait(empty + 8 * stage, turn ^ 1)) {
                    s_fail = 1;
                    break;
                }
                const u32 dst = ring_u + (u32)stage * (u32)stage_bytes;
                mbar_expect(full + 8 * stage, (u32)stage_bytes);
                if (TRANS) tma_load(dst, &P.w, block * PJ_WIDE, g * GROUP, full + 8 * stage);
                else tma_load(dst, &P.w, g * GROUP, block * PJ_WIDE, full + 8 * stage);
                tma_load(dst + PJ_A, &P.x, g * GROUP, (int)row0, full + 8 * stage);
                if (++stage == P.stages) {
                    stage = 0;
                    turn ^= 1;
                }
            }
        }
    } else if (warp == 1) {             // ---- products
        if (lane == 0) {
            const u32 idesc = umma_idesc(TRANS, PJ_WIDE, P.tile);
            const u32 sa = tmem + (u32)P.tile;
            int stage = 0;
            u32 turn = 0;
            bool fine = true;
            for (int q = q0; q < q1 && fine; ++q) {
                const int slot = (q - q0) % PJ_SLOTS;
                const u32 to = sa + (u32)((q - q0) & 1) * 8;
                fine = mbar_wait(sc_full + 8 * slot, (u32)((q - q0) / PJ_SLOTS) & 1);
                if (!fine) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                scales_to_tmem(to, umma_desc(scales_u + (u32)slot * PJ_SCALES, 128, 0));
                scales_to_tmem(to + 4, umma_desc(scales_u + (u32)slot * PJ_SCALES + 512, 128, 0));
                for (int g = q * PJ_QUAD; g < min((q + 1) * PJ_QUAD, g1); ++g) {
                    fine = mbar_wait(full + 8 * stage, turn);
                    if (!fine) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const u32 src = ring_u + (u32)stage * (u32)stage_bytes;
                    const u64 a = umma_desc(src, 1024, 2), b = umma_desc(src + PJ_A, 1024, 2);
                    const u32 id = umma_idesc_at(idesc, (u32)(g % PJ_QUAD));
#pragma unroll
                    for (int k = 0; k < 4; ++k)         // (32 of the depth: 32 bytes within the swizzled rows, or 32 rows)
                        umma_scaled(tmem, a + (TRANS ? k * (32 * GROUP / 16) : k * 2), b + k * 2, id, to, to + 4, g > g0 || k > 0);
                    umma_commit(empty + 8 * stage);
                    if (++stage == P.stages) {
                        stage = 0;
                        turn ^= 1;
                    }
                }
                if (fine) umma_commit(sc_empty + 8 * slot);
            }
            if (!fine) s_fail = 1;
            umma_commit(done);
        }
    } else if (warp == 2) {             // ---- scales
        u32 wa = 0, wx[4];
        auto fetch = [&](int q) {
            wa = weight_scales(P, q, block);
#pragma unroll
            for (int c = 0; c < 4; ++c) wx[c] = c * 32 < P.tile ? row_scales(P, q, row0 + c * 32 + lane) : 0u;
        };
        if (q0 < q1) fetch(q0);
        for (int q = q0; q < q1; ++q) {
            const int i = q - q0, slot = i % PJ_SLOTS;
            if (i >= PJ_SLOTS && !mbar_wait(sc_empty + 8 * slot, (u32)(i / PJ_SLOTS - 1) & 1)) {
                s_fail = 1;
                break;
            }
            uint4 *to = reinterpret_cast<uint4 *>(scales + slot * PJ_SCALES) + lane;
            to[0] = make_uint4(wa, wa, wa, wa);
            to[32] = make_uint4(wx[0], wx[1], wx[2], wx[3]);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(sc_full + 8 * slot);
            if (q + 1 < q1) fetch(q + 1);
        }
    }
    __syncwarp();
    bool fine = mbar_wait(done, 0);
    __syncthreads();
    fine = fine && !s_fail;
    if (!fine && tid == 0) {            // a wait ran out: the results are no numbers, but no copy lands in what comes next
        const int n = g1 - g0;
        for (int i = max(0, n - P.stages); i < n; ++i) mbar_wait(full + 8 * (i % P.stages), (u32)(i / P.stages) & 1);
    }
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    float *sums = reinterpret_cast<float *>(ring);                      // [row][128 output columns]
    for (int c = 0; c < P.tile; c += 16) {
        float v[16];
        tmem_ld(tmem + ((u32)warp << 21) + (u32)c, v);
        tmem_ld_wait(v);
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[(c + i) * PJ_WIDE + tid] = !fine ? __uint_as_float(0x7FFFFFFFu) : q0 < q1 ? v[i] : 0.0f;
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 3) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(P.columns) : "memory");
    }
    if (parts > 1) cluster.sync();
    const int r0 = P.tile * part / parts, r1 = P.tile * (part + 1) / parts;
    const int col = block * PJ_WIDE + tid % 16 * 8;
    for (int r = r0 + tid / 16; r < r1; r += 8) {
        if (row0 + r >= P.rows) break;
        float v[8] = {};
        for (int p = 0; p < parts; ++p) {
            const float4 *s = reinterpret_cast<const float4 *>((parts > 1 ? cluster.map_shared_rank(sums, p) : sums) + r * PJ_WIDE + tid % 16 * 8);
            const float4 x = s[0], y = s[1];
            v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
            v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
        }
        Eight<T> e;
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = from_f32<T>(v[i]);
        T *out = (T *)P.out + (row0 + r) * P.ldo;
        if (P.access == 8) store8<8>(out, col, P.width, e);
        else if (P.access == 4) store8<4>(out, col, P.width, e);
        else store8<1>(out, col, P.width, e);
    }
    if (parts > 1) cluster.sync();      // (nobody leaves while its sums are read)
}

}  // namespace cs
