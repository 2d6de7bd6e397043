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
#include "projection_cut.h"
#include "ring.h"

namespace cs {

static_assert(PJ_GROUP == GROUP, "columns that share a scale");
constexpr int PJ_STAGES = 12;           // most stages of the ring
// Two warps bring the scales, two quads at a time and in turn: a warp's loads for its next two are on their way while it waits for
// room. (One warp, a quad at a time, kept the products waiting: 2.2 PFLOP/s.)
// A slot is a place in shared memory and one in tensor memory: it is filled again when the products of its batch are complete.
constexpr int PJ_BATCH = 2, PJ_SLOTS = 2 * PJ_BATCH;    // quads
constexpr int PJ_SCALES = 1024;         // bytes of a quad's scales: weights, rows
constexpr int PJ_PAD = 1024;            // swizzle patterns start at multiples of 1024 bytes

struct ProjectionParams {
    CUtensorMap w, x;                   // codes, boxes of 128 bytes x 128 resp. `tile` rows
    const u8 *w_scales, *x_scales;
    long long w_depth, w_wide;          // distance of the weights' scales by group of the depth, by 128 output columns
    long long ld_xs, ldo;
    void *out;
    long long rows;
    int width, groups;                  // output columns, groups of the depth
    int blocks;                         // of 128 output columns; of pairs: of 256
    int tiles;                          // pairs: tiles in all
    int tile;                           // rows of a tile, a multiple of 16
    int stages, ring;                   // ring: bytes of the stages, or of the sums that lie there in the end
    int access;                         // values of a row of the result that may be written at once
    u32 columns;                        // of tensor memory
};

__device__ __forceinline__ u32 smem_u32(const void *p) { return (u32)__cvta_generic_to_shared(p); }
// One lane of a warp whose lanes are all here. The compiler knows the region behind it for a single thread's, which a comparison of the
// lane's number does not tell it: products alone, 128 rows, went from 230 to 160 ns for a group of the depth.
__device__ __forceinline__ bool elect_one()
{
    u32 p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
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
template <int N>
__device__ __forceinline__ void tmem_ld_wait(float (&v)[N])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+f"(v[i]));          // (no use of the values may move ahead of the wait)
}

// The scale bytes of a quad on their way to shared memory: those of 128 output columns' weights, the same for all of them, and
// those of the rows `lane`, `lane` + 32, ... of a tile. Nothing here is looked at before it is stored, so that all loads leave together. Bytes
// that fill up a row's last word are not scales and are not read. Of three that are left there the third is another load: by pairs, which take
// tile after tile, it is kept apart (8000 rows 300 -> 8000: 42.6 us, joined at once 46.8), by a CTA with one tile it is joined at once (32 rows
// 6000 -> 1500: 7.9 us, kept apart 8.2).
template <int N>
struct QuadScales {
    static constexpr bool APART = N > 4;
    u32 w[PJ_QUAD], x[N], third[N];

    __device__ __forceinline__ void fetch(const ProjectionParams &P, int quad, long long block, long long row)
    {
        const u8 *s = P.w_scales + min(block, (long long)(P.width - 1) / GROUP) * P.w_wide;
        const int g = quad * PJ_QUAD, left = P.groups - g;
#pragma unroll
        for (int b = 0; b < PJ_QUAD; ++b) w[b] = s[min(g + b, P.groups - 1) * P.w_depth];       // (past the last group: anything, it is not used)
#pragma unroll
        for (int c = 0; c < N; ++c) {
            third[c] = 0;
            if (c * 32 < P.tile) {
                const long long r = min(row + c * 32, P.rows - 1);      // (past the last row: the same)
                const u8 *at = P.x_scales + r * P.ld_xs + g;
                if (left >= PJ_QUAD) {
                    x[c] = *reinterpret_cast<const u32 *>(at);
                } else {
                    x[c] = left >= 2 ? *reinterpret_cast<const u16 *>(at) : at[0];
                    if (left == 3) {
                        if (APART) third[c] = at[2];
                        else x[c] |= (u32)at[2] << 16;
                    }
                }
            } else {
                x[c] = 0;
            }
        }
    }
    // 512 bytes for the weights, 512 for each 128 rows: 32 lanes of four words
    __device__ __forceinline__ void store(char *to, int lane) const
    {
        const u32 a = w[0] | w[1] << 8 | w[2] << 16 | w[3] << 24;
        uint4 *d = reinterpret_cast<uint4 *>(to) + lane;
        d[0] = make_uint4(a, a, a, a);
        const auto row = [&](int c) { return c < N ? x[c < N ? c : 0] | third[c < N ? c : 0] << 16 : 0u; };
#pragma unroll
        for (int i = 0; i < (N + 3) / 4; ++i) d[32 * (i + 1)] = make_uint4(row(4 * i), row(4 * i + 1), row(4 * i + 2), row(4 * i + 3));
    }
};

// (of rows that allow four values at once, at least)
template <class T>
__device__ __forceinline__ void store_result(const ProjectionParams &P, long long row, int col, const Eight<T> &e)
{
    T *out = (T *)P.out + row * P.ldo;
    if (P.access == 8) store8<8>(out, col, P.width, e);
    else store8<4>(out, col, P.width, e);
}

// Sums of rows r0 .. r1 - 1 of a tile over `parts` CTAs of the cluster (every `step`th from `first` on), in their order, into the result.
// The loads of all parts, and of two rows, leave together: one after the other they took 10 us for four parts.
template <class T, int THREADS_>
__device__ __forceinline__ void add_parts(const ProjectionParams &P, cooperative_groups::cluster_group &cluster, float *sums, int parts, int first, int step, bool fine,
                                          long long row0, int r0, int r1, int col0)
{
    constexpr int AHEAD = 4, ROWS = THREADS_ / 16;
    const int c = threadIdx.x % 16 * 8;
    r1 = (int)min((long long)r1, P.rows - row0);
    if (P.access == 1) {                // results column by column, so that neighbouring lanes write neighbours
        constexpr int N = 4, STEP = THREADS_ / PJ_WIDE;
        const int column = threadIdx.x % PJ_WIDE;
        for (int r = r0 + (int)threadIdx.x / PJ_WIDE; r < r1; r += N * STEP) {
            float v[N];
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = fine ? 0.0f : __uint_as_float(0x7FFFFFFFu);
            for (int p = 0; p < parts; ++p) {
                const float *at = (parts > 1 ? cluster.map_shared_rank(sums, first + p * step) : sums) + column;
                float x[N];
#pragma unroll
                for (int k = 0; k < N; ++k) x[k] = at[min(r + k * STEP, r1 - 1) * PJ_WIDE];
#pragma unroll
                for (int k = 0; k < N; ++k) v[k] += x[k];
            }
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (r + k * STEP < r1 && col0 + column < P.width) ((T *)P.out)[(row0 + r + k * STEP) * P.ldo + col0 + column] = from_f32<T>(v[k]);
        }
        return;
    }
    for (int r = r0 + (int)threadIdx.x / 16; r < r1; r += 2 * ROWS) {
        float v[2][8];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = fine ? 0.0f : __uint_as_float(0x7FFFFFFFu);
        for (int p = 0; p < parts; p += AHEAD) {
            float4 x[AHEAD][2][2];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
                if (p + j < parts) {
                    const float *at = (parts > 1 ? cluster.map_shared_rank(sums, first + (p + j) * step) : sums) + c;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        if (r + k * ROWS < r1) {
                            x[j][k][0] = *reinterpret_cast<const float4 *>(at + (r + k * ROWS) * PJ_WIDE);
                            x[j][k][1] = *reinterpret_cast<const float4 *>(at + (r + k * ROWS) * PJ_WIDE + 4);
                        }
                }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
                if (p + j < parts)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        v[k][0] += x[j][k][0].x; v[k][1] += x[j][k][0].y; v[k][2] += x[j][k][0].z; v[k][3] += x[j][k][0].w;
                        v[k][4] += x[j][k][1].x; v[k][5] += x[j][k][1].y; v[k][6] += x[j][k][1].z; v[k][7] += x[j][k][1].w;
                    }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (r + k * ROWS < r1) {
                store_result<T>(P, row0 + r + k * ROWS, col0 + c, rounded<T>(v[k]));
            }
    }
}

// A cluster of CTAs takes a tile: its CTAs share the depth by quads, each leaves its sums in its own shared memory, and
// each adds up a part of the tile's rows over all of them, in their order, by distributed shared memory. (Sending the sums to where they
// are added, into room of their own, spared a barrier and took 1 to 7 us more.)
// Four warps: copies, products, and two for the scales; then all take the sums.
// Bound by launch, first copies and the end (3.4 us for 1 row 512 -> 512), then by the codes on their way: 1 row 1500 -> 6000: 5.2 us
// (1.4 for 9 MB); 1 row 9216^2: 17.0 us (13.0), 4096 -> 33278: 23.0 us (20.9); 64 rows 9216 -> 4096: 13.6 us (5.9). All shared memory for the
// ring where the CTAs are no more than SMs, since what is under way hides the latency (64 rows 9216 -> 4096 with half of it: 15.4 us).
template <class T, bool TRANS>
__global__ void __launch_bounds__(128, 2) k_projection(const __grid_constant__ ProjectionParams P)
{
    extern __shared__ char pj_raw[];
    __shared__ u64 bars[2 * PJ_STAGES + 4 + 1];
    __shared__ u32 s_tmem;
    __shared__ int s_fail, s_issued;
    char *ring = pj_raw + ((PJ_PAD - (smem_u32(pj_raw) & (PJ_PAD - 1))) & (PJ_PAD - 1));
    char *scales = ring + P.ring;
    const u32 ring_u = smem_u32(ring), scales_u = smem_u32(scales);
    const u32 full = smem_u32(bars), empty = full + 8 * PJ_STAGES, sc_full = empty + 8 * PJ_STAGES, sc_empty = sc_full + 16,
              done = sc_empty + 16;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
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
        for (int s = 0; s < 2; ++s) {
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
        if (elect_one()) {
            int stage = 0, g = g0;
            u32 turn = 0;
            for (; g < g1; ++g) {
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
            s_issued = g - g0;
        }
    } else if (warp == 1) {             // ---- products
        if (elect_one()) {
            const u32 idesc = umma_idesc(TRANS, PJ_WIDE, P.tile);
            const u32 sa = tmem + (u32)P.tile;
            int stage = 0;
            u32 turn = 0;
            bool fine = true;
            for (int q = q0; q < q1 && fine; ++q) {
                const int i = q - q0, slot = i % PJ_SLOTS, batch = i / PJ_BATCH;
                const u32 to = sa + (u32)slot * 8;
                if (i % PJ_BATCH == 0) {
                    fine = mbar_wait(sc_full + 8 * (batch & 1), (u32)(batch / 2) & 1);
                    if (!fine) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                }
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
                if (fine && i % PJ_BATCH == PJ_BATCH - 1) umma_commit(sc_empty + 8 * (batch & 1));
            }
            if (!fine) s_fail = 1;
            umma_commit(done);
        }
    } else {                            // ---- scales
        const int side = warp - 2;
        QuadScales<4> next[PJ_BATCH];
        auto fetch = [&](int q) {
#pragma unroll
            for (int j = 0; j < PJ_BATCH; ++j)
                if (q + j < q1) next[j].fetch(P, q + j, block, row0 + lane);
        };
        int q = q0 + side * PJ_BATCH;
        fetch(q);
        for (u32 turn = 0; q < q1; q += PJ_SLOTS, turn ^= 1) {
            if (q >= q0 + PJ_SLOTS && !mbar_wait(sc_empty + 8 * side, turn ^ 1)) {
                s_fail = 1;
                break;
            }
#pragma unroll
            for (int j = 0; j < PJ_BATCH; ++j)
                if (q + j < q1) next[j].store(scales + (side * PJ_BATCH + j) * PJ_SCALES, lane);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(sc_full + 8 * side);
            fetch(q + PJ_SLOTS);
        }
    }
    __syncwarp();
    bool fine = mbar_wait(done, 0);     // (the last commit of the thread whose commits arrive here: those ahead of it are through)
    __syncthreads();
    fine = fine && !s_fail;
    if (!fine && tid == 0)              // a wait ran out: the results are no numbers, but no copy lands in what comes next
        copies_under_way(s_issued, P.stages, [&](int s, int parity) { mbar_wait(full + 8 * s, (u32)parity); });
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
    add_parts<T, 128>(P, cluster, sums, parts, 0, 1, true, row0, P.tile * part / parts, P.tile * (part + 1) / parts, block * PJ_WIDE);
    if (parts > 1) cluster.sync();      // (nobody leaves while its sums are read)
}

// ------------------------------------------------------------------ many rows: pairs of CTAs
// Two CTAs of a cluster form one product of 256 output columns (tcgen05 cta_group::2): each brings its own 128 columns of
// weights and half of the rows, and keeps its 128 columns' sums; per byte that an SM takes from L2 this is up to 1.87 times the work
// of a CTA by itself (224 rows in 30 KB for a group of the depth, 128 rows in 32 KB). The first CTA of the pair issues the products.
// Persistent: two accumulators in tensor memory take turns, so that a tile is written out while the next one is multiplied. SPLIT: the
// pairs of a cluster share one tile's depth instead, as in the kernel above.
// Bound by the tensor core (86 % of its cycles at 6011 rows 9216 -> 4096) and by what the tiles take from L2:
// 152 us, 2.99 PFLOP/s, back to back; 8192 rows 4096^2 backward 94 us, 2.91 PFLOP/s. (The products alone, with no copies, take 3.7 PFLOP/s;
// 5 to 7 stages and any L2 promotion are alike.) 700 rows 1500 <- 33278: 46.4 us with rows of codes 1504 bytes apart, 44.3 with 1536 (a
// 128-byte piece of a row that starts anywhere is two lines); 1504 columns, whose results go by eights, 39.7, 1536 columns 34.6.
constexpr int PP_OUT_WARPS = 8;         // warps that write results: two for each 32 lanes of tensor memory, in turn
constexpr int PP_THREADS = 128 + 32 * PP_OUT_WARPS;
constexpr int PP_STAGES = 8;
constexpr int PP_SCALES = 1536;         // bytes of a quad's scales: weights, rows
constexpr int PP_COLUMNS = 512;
constexpr int PP_OUT = PP_OUT_WARPS * 2048;     // where they turn their sums around

__device__ __forceinline__ u32 peer_address(u32 addr, u32 rank)
{
    u32 r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// An arrival at a barrier of any CTA of the cluster, of CTA scope. Nothing is carried from one CTA to the other by it: the scales that it announces are
// read by the tensor core of the CTA that wrote them, behind a fence for that in the thread that wrote them; an accumulator that it gives back has
// been read. That this order holds for products that the other CTA issues is the hardware's doing (an arrival leaves an SM behind the shared-memory
// writes ahead of it), not a promise of PTX's scopes, which ask for release and acquire at cluster scope; a part that reorders the two would need
// them. They cost each launch 0.9 us (512 rows of 4096^2: 12.3 instead of 11.4 us, 128 rows 10.5 instead of 9.6).
__device__ __forceinline__ void mbar_arrive_at(u32 cluster_addr) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" :: "r"(cluster_addr) : "memory"); }
// A box into this CTA's shared memory, counted at a barrier of either CTA of the pair.
__device__ __forceinline__ void tma_load_pair(u32 dst, const CUtensorMap *map, int x, int y, u32 bar)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void umma_scaled_pair(u32 d, u64 a, u64 b, u32 idesc, u32 scale_a, u32 scale_b, u32 add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\ttcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(scale_a), "r"(scale_b), "r"(add) : "memory");
}
// Each CTA's scales, from its own shared memory into its own tensor memory.
__device__ __forceinline__ void scales_to_tmem_pair(u32 tmem, u64 desc)
{
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" :: "r"(tmem), "l"(desc) : "memory");
}
// Arrives at the barrier of this address in both CTAs once the products so far are done.
__device__ __forceinline__ void umma_commit_pair(u32 bar, u32 ranks)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" :: "r"(bar), "h"((u16)ranks) : "memory");
}
__device__ __forceinline__ void tmem_ld(u32 addr, float (&v)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
                   "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]),
                   "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]),
                   "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31]) : "r"(addr));
}
// Sums of 32 rows x 32 output columns, a column per lane, into the result: neighbouring rows go as pairs through the
// warp's 2 KB of shared memory and come back as eight neighbouring columns of a row. `out`: row 0, column 0; `rows` of them are wanted.
template <int A, class T>
__device__ __forceinline__ void write_block(const float (&v)[32], u32 *turn, T *out, long long ldo, int rows, int col0, int width, int lane)
{
    if constexpr (A == 1) {             // (neighbouring columns are neighbouring lanes' already)
        if (col0 + lane < width)
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i < rows) out[i * ldo + col0 + lane] = from_f32<T>(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) turn[i * 32 + lane] = pack2(v[2 * i], v[2 * i + 1], T());
        __syncwarp();
        const int i0 = lane / 4, n8 = lane % 4 * 8, first = (i0 & 1) * 4;      // (odd pairs read their halves the other way round: no bank conflicts)
        T *row = out + (long long)(2 * i0) * ldo;
#pragma unroll
        for (int r = 0; r < 2; ++r, row += 16 * ldo) {
            const u32 *at = turn + (r * 8 + i0) * 32 + n8;
            const uint4 x = *reinterpret_cast<const uint4 *>(at + first), y = *reinterpret_cast<const uint4 *>(at + (4 - first));
            const uint4 a = first ? y : x, b = first ? x : y;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32 sel = h ? 0x7632u : 0x5410u;
                Eight<T> e;
                *reinterpret_cast<uint4 *>(&e) = make_uint4(__byte_perm(a.x, a.y, sel), __byte_perm(a.z, a.w, sel), __byte_perm(b.x, b.y, sel), __byte_perm(b.z, b.w, sel));
                if (16 * r + 2 * i0 + h < rows) store8<A>(row + h * ldo, col0 + n8, width, e);
            }
        }
        __syncwarp();
    }
}

template <class T, bool TRANS, bool SPLIT>
__global__ void __launch_bounds__(PP_THREADS, 1) k_projection_pair(const __grid_constant__ ProjectionParams P)
{
    extern __shared__ char pj_raw[];
    __shared__ u64 bars[2 * PP_STAGES + 4 + 4];
    __shared__ u32 s_tmem;
    __shared__ int s_fail;
    char *ring = pj_raw + ((PJ_PAD - (smem_u32(pj_raw) & (PJ_PAD - 1))) & (PJ_PAD - 1));
    char *scales = ring + P.ring, *turn_room = scales + PJ_SLOTS * PP_SCALES;
    const u32 ring_u = smem_u32(ring), scales_u = smem_u32(scales);
    const u32 full = smem_u32(bars), empty = full + 8 * PP_STAGES, sc_full = empty + 8 * PP_STAGES, sc_empty = sc_full + 16,
              acc_full = sc_empty + 16, acc_empty = acc_full + 16;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const u32 rank = cluster.block_rank(), side = rank & 1, leader = rank & ~1u, both = 3u << leader;
    const int parts = SPLIT ? (int)cluster.num_blocks() / 2 : 1, part = SPLIT ? (int)rank / 2 : 0;
    const u32 tiles = (u32)P.tiles, first = SPLIT ? blockIdx.x / (2 * parts) : blockIdx.x / 2, stride = SPLIT ? tiles : gridDim.x / 2;
    const int quads = (P.groups + PJ_QUAD - 1) / PJ_QUAD, q0 = (int)((long long)quads * part / parts), q1 = (int)((long long)quads * (part + 1) / parts);
    const int g0 = q0 * PJ_QUAD, g1 = min(q1 * PJ_QUAD, P.groups);
    const int half = P.tile / 2, stage_bytes = PJ_A + half * GROUP;

    if (tid == 0) {
        asm volatile("prefetch.tensormap [%0];" :: "l"(&P.w) : "memory");
        asm volatile("prefetch.tensormap [%0];" :: "l"(&P.x) : "memory");
        for (int s = 0; s < PP_STAGES; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(sc_full + 8 * s, 2);
            mbar_init(sc_empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(acc_full + 8 * s, 1);
            mbar_init(acc_empty + 8 * s, 2 * PP_OUT_WARPS);
        }
        s_fail = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 3) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&s_tmem)), "r"(PP_COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster.sync();                     // (the barriers of both CTAs are there)
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const u32 tmem = s_tmem;
    pdl_wait();
    pdl_launch_dependents();

    if (warp == 0) {                    // ---- copies, in both CTAs; counted at the leader's barriers
        if (elect_one()) {
            const u32 full_at = peer_address(full, leader);
            int stage = 0, issued = 0;
            u32 turn = 0;
            bool fine = true;
            for (u32 t = first; t < tiles && fine; t += stride) {
                const int col = (int)(t % (u32)P.blocks * 2 + side) * PJ_WIDE, row = (int)(t / (u32)P.blocks) * P.tile + (int)side * half;
                for (int g = g0; g < g1; ++g) {
                    if (issued >= P.stages) fine = mbar_wait(empty + 8 * stage, turn ^ 1);
                    if (!fine) break;
                    ++issued;
                    const u32 dst = ring_u + (u32)stage * (u32)stage_bytes, bar = full_at + 8 * stage;
                    if (side == 0) mbar_expect(full + 8 * stage, 2 * (u32)stage_bytes);
                    if (TRANS) tma_load_pair(dst, &P.w, col, g * GROUP, bar);
                    else tma_load_pair(dst, &P.w, g * GROUP, col, bar);
                    tma_load_pair(dst + PJ_A, &P.x, g * GROUP, row, bar);
                    if (++stage == P.stages) {
                        stage = 0;
                        turn ^= 1;
                    }
                }
            }
            // The leader's commits arrive in both CTAs: each is waited for before a CTA ends. (Nobody waits for this: the products are behind it.)
            copies_under_way(issued, P.stages, [&](int s, int parity) { fine = fine && mbar_wait(empty + 8 * s, (u32)parity); });
            if (!fine) {                // a wait ran out, here or in a warp that this one heard no more of: the results are no numbers
                s_fail = 1;
                // No copy lands in what comes next: the leader, at whose barriers both CTAs' copies are counted, waits for all of them
                // ahead of the cluster's last barrier.
                if (side == 0) copies_under_way(issued, P.stages, [&](int s, int parity) { mbar_wait(full + 8 * s, (u32)parity); });
            }
        }
    } else if (warp == 1) {             // ---- products, issued by the leader
        if (side == 0 && elect_one()) {
            const u32 idesc = umma_idesc(TRANS, 2 * PJ_WIDE, P.tile), sa = tmem + 2 * (u32)P.tile;
            int stage = 0, quad = 0, done = 0;
            u32 turn = 0;
            bool fine = true;
            for (u32 t = first; t < tiles && fine; t += stride, ++done) {
                const u32 buf = (u32)done & 1, d = tmem + buf * (u32)P.tile;
                if (done >= 2) fine = mbar_wait(acc_empty + 8 * buf, (u32)(done / 2 - 1) & 1);
                if (!fine) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (int q = q0; q < q1 && fine; ++q, ++quad) {
                    const u32 slot = (u32)quad % PJ_SLOTS, to = sa + slot * 12, src = scales_u + slot * PP_SCALES, batch = (u32)quad / PJ_BATCH;
                    if (quad % PJ_BATCH == 0) {
                        fine = mbar_wait(sc_full + 8 * (batch & 1), batch / 2 & 1);
                        if (!fine) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    }
#pragma unroll
                    for (int i = 0; i < 3; ++i) scales_to_tmem_pair(to + 4 * i, umma_desc(src + 512 * i, 128, 0));
                    for (int g = q * PJ_QUAD; g < min((q + 1) * PJ_QUAD, g1); ++g) {
                        fine = mbar_wait(full + 8 * stage, turn);
                        if (!fine) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const u32 at = ring_u + (u32)stage * (u32)stage_bytes;
                        const u64 a = umma_desc(at, 1024, 2), b = umma_desc(at + PJ_A, 1024, 2);
                        const u32 id = umma_idesc_at(idesc, (u32)(g % PJ_QUAD));
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            umma_scaled_pair(d, a + (TRANS ? k * (32 * GROUP / 16) : k * 2), b + k * 2, id, to, to + 4, g > g0 || k > 0);
                        umma_commit_pair(empty + 8 * stage, both);
                        if (++stage == P.stages) {
                            stage = 0;
                            turn ^= 1;
                        }
                    }
                    if (fine && quad % PJ_BATCH == PJ_BATCH - 1) umma_commit_pair(sc_empty + 8 * (batch & 1), both);
                }
                if (fine) umma_commit_pair(acc_full + 8 * buf, both);
            }
            if (!fine) s_fail = 1;
        }
    } else if (warp < 4) {              // ---- scales: each CTA's weights, and all rows'
        const int turns = warp - 2;
        const u32 full_at = peer_address(sc_full + 8 * turns, leader);
        QuadScales<7> next[PJ_BATCH];
        u32 t = first;                  // the quad that is fetched next
        int q = q0;
        auto skip = [&]() {
            if (++q == q1) {
                q = q0;
                t = tiles - t > stride ? t + stride : tiles;
            }
        };
        auto fetch = [&]() {
#pragma unroll
            for (int j = 0; j < PJ_BATCH; ++j)
                if (t < tiles) {
                    next[j].fetch(P, q, (long long)(t % (u32)P.blocks * 2 + side), (long long)(t / (u32)P.blocks) * P.tile + lane);
                    skip();
                }
        };
        auto pass = [&]() {             // (the other warp's)
            for (int j = 0; j < PJ_BATCH; ++j)
                if (t < tiles) skip();
        };
        const long long all = first < tiles ? (long long)((tiles - first + stride - 1) / stride) * (q1 - q0) : 0;
        if (turns) pass();
        fetch();
        u32 phase = 0;
        bool fine = true;
        for (long long i = turns * PJ_BATCH; i < all; i += PJ_SLOTS, phase ^= 1) {
            fine = i < PJ_SLOTS || mbar_wait(sc_empty + 8 * turns, phase ^ 1);
            if (!fine) break;
#pragma unroll
            for (int j = 0; j < PJ_BATCH; ++j)
                if (i + j < all) next[j].store(scales + (turns * PJ_BATCH + j) * PP_SCALES, lane);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive_at(full_at);
            pass();
            fetch();
        }
        if (fine && last_batch_commits(all, PJ_BATCH, turns)) fine = mbar_wait(sc_empty + 8 * turns, phase ^ 1);
        if (!fine) s_fail = 1;
    } else if (warp >= 4) {             // ---- results
        const u32 empty_at = peer_address(acc_empty, leader);
        const int w = warp & 3, turns = (warp - 4) / 4;
        u32 *turn = reinterpret_cast<u32 *>(turn_room + (warp - 4) * 2048);
        bool fine = true;
        int done = 0;
        for (u32 t = first; t < tiles; t += stride, ++done) {
            const u32 buf = (u32)done & 1;
            fine = fine && mbar_wait(acc_full + 8 * buf, (u32)(done / 2) & 1);
            __syncwarp();
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const u32 at = tmem + ((u32)w << 21) + buf * (u32)P.tile;
            const long long row0 = (long long)(t / (u32)P.blocks) * P.tile;
            const int col0 = (int)(t % (u32)P.blocks * 2 + side) * PJ_WIDE + w * 32;
            const int rows = (int)min(P.rows - row0, (long long)P.tile);
#pragma unroll 1
            for (int c = turns * 32; c < P.tile; c += PP_OUT_WARPS / 4 * 32) {          // (the last may be a half: what is behind it is read, not used)
                float v[32];
                tmem_ld(at + (u32)c, v);
                tmem_ld_wait(v);
                if (!fine) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(0x7FFFFFFFu);
                }
                if constexpr (SPLIT) {
                    float *sums = reinterpret_cast<float *>(ring);          // [row][128 output columns]
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (i < 16 || c + 16 < P.tile) sums[(c + i) * PJ_WIDE + w * 32 + lane] = v[i];
                } else if (c < rows) {
                    T *out = (T *)P.out + (row0 + c) * P.ldo;
                    if (P.access == 8) write_block<8>(v, turn, out, P.ldo, rows - c, col0, P.width, lane);
                    else if (P.access == 4) write_block<4>(v, turn, out, P.ldo, rows - c, col0, P.width, lane);
                    else write_block<1>(v, turn, out, P.ldo, rows - c, col0, P.width, lane);
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive_at(empty_at + 8 * buf);          // (its sums are in registers or written)
        }
        if (!fine) s_fail = 1;
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster.sync();                     // (both CTAs are through with their tensor memory and each other's barriers)
    if (warp == 3) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(PP_COLUMNS) : "memory");
    }
    if constexpr (SPLIT) {
        int fail = 0;                   // (of any CTA of the cluster)
        for (int p = 0; p < 2 * parts; ++p) fail |= *cluster.map_shared_rank(&s_fail, p);
        add_parts<T, PP_THREADS>(P, cluster, reinterpret_cast<float *>(ring), parts, (int)side, 2, !fail, (long long)(first / (u32)P.blocks) * P.tile,
                                 P.tile * part / parts, P.tile * (part + 1) / parts, (int)(first % (u32)P.blocks * 2 + side) * PJ_WIDE);
        cluster.sync();                 // (nobody leaves while its sums are read)
    }
}

}  // namespace cs
