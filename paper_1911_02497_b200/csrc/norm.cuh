// Root-mean-square norm of rows with the residual's addition, forward and backward, and the encoders of rows and of blocks.
//
// All of it is bound by memory: a few operations for every 2 to 16 bytes. So each value is read once and kept, as it came, in
// the registers of the threads that share a row (TPR of them, NV times eight neighbouring columns each) while the row's sum
// is formed, and everything that is written leaves in the same pass, codes and scales included: a group of 128 columns
// is 16 neighbouring lanes, its largest magnitude four shuffles.
#pragma once
#include "coded.cuh"
#include "row_runs.h"

namespace cs {

struct NormParams {
    const void *x, *residual, *gain;
    void *h, *y;
    u8 *codes, *scales;
    float *rstd;
    long long ldx, ldr, ldh, ldy, ldc, lds;
    long long rows;
    int cols;
    float inv_cols;                     // 1 / cols
    int gain_f32;
    float eps;
};

struct NormBackParams {
    const void *dy, *dh, *h, *gain;
    const float *rstd;
    void *dx;
    u8 *codes, *scales;
    float *part;                        // [slots][ld_part]: sums for dgain; NULL: not wanted
    long long ldy, ldd, ldh, ldx, ldc, lds, ld_part;
    long long rows;
    int cols;
    float inv_cols;
    int gain_f32;
};

// ------------------------------------------------------------------ sums over a row
template <class F>
__device__ __forceinline__ F lanes_sum(F v, int lanes)
{
    for (int d = lanes / 2; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

// Sum over the TPR threads of a row, the same bits in each. A row of more than one warp is the whole CTA, which passes one
// barrier; `slots` is one of two that take turns, so that nobody writes what another still reads.
template <int TPR, class F>
__device__ __forceinline__ F row_sum(F v, F *slots)
{
    v = lanes_sum(v, 32);
    if (TPR == 32) return v;
    const int lane = threadIdx.x & 31;
    if (lane == 0) slots[threadIdx.x >> 5] = v;
    __syncthreads();
    return lanes_sum(lane < TPR / 32 ? slots[lane] : (F)0, 32);
}

// 1 / sqrt(x), x the mean of squares and eps (the root's approximation, and one Newton step: every thread of a row does this, and quotients and
// roots in full were a tenth of the kernel)
__device__ __forceinline__ float rstd_of(float x)
{
    const float r = rsqrtf(x);
    return fmaf(r * 0.5f, fmaf(-x * r, r, 1.0f), r);
}
// Whether fp32 can be trusted with x: not where it or the squares' sum overflowed or is no number, nor where squares may have been
// subnormal. Each of those lost at most 2^-150, so from 2^-100 on all of them lost less than 2^-50 of x.
__device__ __forceinline__ bool in_fp32_range(float x) { return x >= 0x1p-100f && x <= 3.4e38f; }
__device__ __forceinline__ float rstd_of(double sum, int cols, float eps) { return (float)(1.0 / sqrt(sum / cols + (double)eps)); }

template <class T, int A>
__device__ __forceinline__ void load_gain(const void *gain, int f32, int c, int cols, float (&g)[8])
{
    if (!gain) {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = 1.0f;
    } else if (f32) {
        widen(load8<A>((const float *)gain, c, cols), g);
    } else {
        widen(load8<A>((const T *)gain, c, cols), g);
    }
}

template <class T>
__device__ __forceinline__ void add_rounded(Eight<T> &h, const Eight<T> &r)
{
    float a[8], b[8];
    widen(h, a);
    widen(r, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] += b[i];
    h = rounded<T>(a);
}
// h of columns c .. c+7: x, or the rounded sum of x and the residual.
template <class T, int A>
__device__ __forceinline__ Eight<T> load_h(const NormParams &P, long long row, int c)
{
    Eight<T> h = load8<A>((const T *)P.x + row * P.ldx, c, P.cols);
    if (P.residual) add_rounded(h, load8<A>((const T *)P.residual + row * P.ldr, c, P.cols));
    return h;
}

// What follows from eight values of h.
template <class T, int A>
__device__ __forceinline__ void norm_out(const NormParams &P, long long row, int c, const Eight<T> &h, float rstd, Eight<T> *turn)
{
    float g[8], y[8];
    load_gain<T, A>(P.gain, P.gain_f32, c, P.cols, g);
    widen(h, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = y[i] * rstd * g[i];
    if (P.y) store8_warp<A>((T *)P.y + row * P.ldy, c, P.cols, rounded<T>(y), turn);
    if (P.codes) {
        if (c + 8 > P.cols) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = c + i < P.cols ? y[i] : 0.0f;        // (a row that is no number)
        }
        encode8<A>(y, P.codes + row * P.ldc, P.scales + row * P.lds, c, P.cols);
    }
}

template <int TPR> struct RowThreads {
    static constexpr int BLOCK = TPR == 32 ? 128 : TPR, ROWS = BLOCK / TPR;
};

// Measured (bf16, residual): 8192 x 4096, 16- and 8-bit results 48 us (46 for the bytes); 8000 x 1500, 8-bit results 19 us (13); rows
// that begin anywhere: 8000 x 2047 39 us (23). Bound by memory, and in the last two by instructions (issue slots 70 % taken). A ring of
// rows copied ahead, as in the backward pass, took longer (60 us against 55 then): many CTAs of one row each overlap by themselves.
template <class T, int A, int TPR, int NV>
__global__ void __launch_bounds__(RowThreads<TPR>::BLOCK) k_norm_forward(const __grid_constant__ NormParams P)
{
    __shared__ float slots[32];
    __shared__ double wide[32];
    __shared__ Eight<T> s_turns[Turns<A, T, RowThreads<TPR>::BLOCK>::N];
    Eight<T> *turn = s_turns + (A == 1 ? threadIdx.x / 32 * 32 : 0);
    pdl_wait();
    pdl_launch_dependents();
    constexpr int ROWS = RowThreads<TPR>::ROWS;
    const long long row = ROWS == 1 ? blockIdx.x : (long long)blockIdx.x * ROWS + threadIdx.x / TPR;
    if (row >= P.rows) return;                          // (whole rows of threads: no barrier misses them)
    const int t = ROWS == 1 ? threadIdx.x : threadIdx.x % TPR;
    const long long ox = row * P.ldx, orr = row * P.ldr, last = P.rows - 1;
    Asked<A, T> ax[NV], ar[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        ax[v] = ask8<A>((const T *)P.x, ox, last * P.ldx + P.cols, (v * TPR + t) * 8, P.cols);
        if (P.residual) ar[v] = ask8<A>((const T *)P.residual, orr, last * P.ldr + P.cols, (v * TPR + t) * 8, P.cols);
    }
    Eight<T> h[NV];
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        h[v] = take8<A>(ax[v], (const T *)P.x, ox, (v * TPR + t) * 8, P.cols);
        if (P.residual) add_rounded(h[v], take8<A>(ar[v], (const T *)P.residual, orr, (v * TPR + t) * 8, P.cols));
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if (P.h) store8_warp<A>((T *)P.h + row * P.ldh, (v * TPR + t) * 8, P.cols, h[v], turn);
        float f[8];
        widen(h[v], f);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(f[i], f[i], sum);
    }
    sum = row_sum<TPR>(sum, slots);
    const float mean = fmaf(sum, P.inv_cols, P.eps);
    float rstd = rstd_of(mean);
    if (!in_fp32_range(mean)) {                         // (the same for the row)
        double d = 0.0;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) d += (double)h[v][i] * h[v][i];
        rstd = rstd_of(row_sum<TPR>(d, wide), P.cols, P.eps);
    }
    if (t == 0 && P.rstd) P.rstd[row] = rstd;
    if (!P.y && !P.codes) return;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        hold(h[v]);
        norm_out<T, A>(P, row, (v * TPR + t) * 8, h[v], rstd, turn);
    }
}

// Rows that are longer than the threads' registers: read twice, the second time mostly from L2.
template <class T, int A, int TPR>
__global__ void __launch_bounds__(TPR) k_norm_forward_long(const __grid_constant__ NormParams P)
{
    __shared__ double slots[32];
    __shared__ Eight<T> s_turns[Turns<A, T, TPR>::N];
    Eight<T> *turn = s_turns + (A == 1 ? threadIdx.x / 32 * 32 : 0);
    pdl_wait();
    pdl_launch_dependents();
    const long long row = blockIdx.x;
    double sum = 0.0;
    for (int c0 = 0; c0 < P.cols; c0 += TPR * 8) {                  // (all lanes stay for the shuffles)
        const int c = c0 + threadIdx.x * 8;
        const Eight<T> h = load_h<T, A>(P, row, c);
        if (P.h) store8_warp<A>((T *)P.h + row * P.ldh, c, P.cols, h, turn);
        double part = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) part += (double)h[i] * h[i];
        sum += part;
    }
    const float rstd = rstd_of(row_sum<TPR>(sum, slots), P.cols, P.eps);
    if (threadIdx.x == 0 && P.rstd) P.rstd[row] = rstd;
    if (!P.y && !P.codes) return;
    for (int c0 = 0; c0 < P.cols; c0 += TPR * 8) {
        const int c = c0 + threadIdx.x * 8;
        // what this thread wrote to h, or x and the residual again where there is no h
        const Eight<T> h = P.h ? load8<A>((const T *)P.h + row * P.ldh, c, P.cols) : load_h<T, A>(P, row, c);
        norm_out<T, A>(P, row, c, h, rstd, turn);
    }
}

// ------------------------------------------------------------------ backward
// dx of columns c .. c+7; q: the mean that is taken out.
template <class T, int A>
__device__ __forceinline__ void norm_back_out(const NormBackParams &P, long long row, int c, const Eight<T> &dy, const Eight<T> &h,
                                              const Eight<T> &dh, const float (&g)[8], float rstd, float q, Eight<T> *turn)
{
    float d[8], u[8], s[8];
    widen(dy, d);
    widen(h, u);
    if (P.dh) widen(dh, s);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        d[i] = rstd * fmaf(-(u[i] * rstd), q, d[i] * g[i]);
        if (P.dh) d[i] += s[i];
    }
    if (P.dx) store8_warp<A>((T *)P.dx + row * P.ldx, c, P.cols, rounded<T>(d), turn);
    if (P.codes) {
        if (c + 8 > P.cols) {
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = c + i < P.cols ? d[i] : 0.0f;
        }
        encode8<A>(d, P.codes + row * P.ldc, P.scales + row * P.lds, c, P.cols);
    }
}

// Operands on their way: the threads of a row copy it into a ring of rows in shared memory (cp.async), so what is in flight does not go by
// registers, and the operands are read from there twice instead of being kept across the row's sum. With loads into registers,
// a row at a time: 91 us for 8192 x 4096 in bf16, against 46 for the bytes. A thread copies the eights that it will use itself, and nobody
// waits for anybody's copies. Where rows begin anywhere (A = 1) it copies the aligned 16 bytes in which its eight begins, one piece more
// ends the row, the row's threads meet, and an eight is shifted together from its pieces (8000 x 2047: 54 us, value by value 155).
template <class T, int A, int TPR, int NV> struct BackRing {
    static constexpr int BLOCK = RowThreads<TPR>::BLOCK, ROWS = RowThreads<TPR>::ROWS, EIGHT = 8 * sizeof(T);
    static constexpr int ROOM = NV * TPR * EIGHT + (A == 1 ? 16 : 0);  // bytes of a row's operand
    static constexpr int STAGE = 3 * ROWS * ROOM;                      // dy, h, dh
    static constexpr int STAGES = 3 * STAGE <= 75 * 1024 ? 3 : 2;
    static constexpr int SMEM = STAGES * STAGE;
    static constexpr int FIT = 226 * 1024 / (SMEM + (A == 1 ? BLOCK * EIGHT : 0) + 2048), WANT = 768 / BLOCK > 0 ? 768 / BLOCK : 1;
    static constexpr int CTAS = FIT < WANT ? FIT : WANT;               // of an SM
    static_assert(SMEM <= 226 * 1024 && CTAS >= 1, "shared memory");
};

// The first `bytes` of 16 (or 8); zeros behind them.
template <int BYTES>
__device__ __forceinline__ void copy_async(u32 dst, const void *src, int bytes)
{
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(bytes) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" :: "r"(dst), "l"(src), "r"(bytes) : "memory");
}
template <int A, class T>
__device__ __forceinline__ void copy8(u32 dst, const T *row, int c, int cols)
{
    constexpr int BYTES = A == 8 || sizeof(T) == 4 ? 16 : 8, N = 8 * sizeof(T) / BYTES, EACH = BYTES / sizeof(T);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool there = c + i * EACH < cols;
        copy_async<BYTES>(dst + i * BYTES, there ? row + c + i * EACH : row, there ? BYTES : 0);
    }
}
// Values that `row` begins behind an aligned 16 bytes.
template <class T> __device__ __forceinline__ int begins_by(const T *row) { return (int)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T)); }
// Piece i of a row that begins anywhere: the aligned 16 bytes that hold its values from i * V - by on. A piece may reach into the
// neighbouring rows, but not out of the matrix (`off`: where the row begins in it, `total`: where it ends).
template <class T>
__device__ __forceinline__ void copy_piece(char *dst, const T *base, long long off, long long total, int i, int cols)
{
    constexpr int V = 16 / (int)sizeof(T);
    const int by = begins_by(base + off), first = i * V - by;
    if (first >= cols) return;
    const long long start = off + first;
    if (start >= 0) {
        copy_async<16>((u32)__cvta_generic_to_shared(dst), base + start, (int)min((long long)V, total - start) * (int)sizeof(T));
    } else {                            // the matrix begins within this piece
        for (int j = 0; j < V; ++j)
            if (start + j >= 0 && start + j < total) reinterpret_cast<T *>(dst)[j] = base[start + j];
    }
}
// The eight at columns c .. c+7 of such a row, whose pieces lie at `room`; zero past its end.
template <class T>
__device__ __forceinline__ Eight<T> from_pieces(const char *room, int by, int c, int cols)
{
    constexpr int W = (int)sizeof(T) * 2;               // words of an eight
    u32 w[W + 4];
    const uint4 *p = reinterpret_cast<const uint4 *>(room + c * (int)sizeof(T));
#pragma unroll
    for (int i = 0; i < W / 4 + 1; ++i) {
        const uint4 x = p[i];
        w[4 * i] = x.x;
        w[4 * i + 1] = x.y;
        w[4 * i + 2] = x.z;
        w[4 * i + 3] = x.w;
    }
    shift_words(w, by);
    Eight<T> e;
    u32 *d = reinterpret_cast<u32 *>(&e);
#pragma unroll
    for (int i = 0; i < W; ++i) d[i] = w[i];
    if (c + 8 > cols) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i >= cols) e.v[i] = from_f32<T>(0.0f);
    }
    return e;
}

// A CTA takes every gridDim-th row (group of rows), so that a thread's sums for dgain stay in its registers; they leave
// once, as one of the slots that k_norm_dgain adds up. Measured with it: 8192 x 4096 bf16, dh and codes, 55 us (46 for the bytes), bound by
// memory (59 % of its nominal rate) and instructions (67 % of the issue slots); 8192 x 1500 28 us (15).
template <class T, int A, int TPR, int NV>
__global__ void __launch_bounds__(RowThreads<TPR>::BLOCK, BackRing<T, A, TPR, NV>::CTAS) k_norm_backward(const __grid_constant__ NormBackParams P)
{
    using R = BackRing<T, A, TPR, NV>;
    constexpr int ROWS = R::ROWS, BLOCK = R::BLOCK, S = R::STAGES;
    extern __shared__ __align__(16) char nb_ring[];
    __shared__ float slots[2][32];
    __shared__ Eight<T> s_turns[Turns<A, T, BLOCK>::N];
    Eight<T> *turn = s_turns + (A == 1 ? threadIdx.x / 32 * 32 : 0);
    pdl_wait();
    pdl_launch_dependents();
    const int t = ROWS == 1 ? threadIdx.x : threadIdx.x % TPR, sub = ROWS == 1 ? 0 : threadIdx.x / TPR;
    constexpr bool KEEP = TPR < 1024;                   // (a thread of 1024 has 64 registers: the gain is read again, from L1)
    float g[NV][8], acc[NV][8] = {};
#pragma unroll
    for (int v = 0; v < NV; ++v)
        if (KEEP) load_gain<T, A>(P.gain, P.gain_f32, (v * TPR + t) * 8, P.cols, g[v]);
    const long long first = (long long)blockIdx.x * ROWS + sub, step = (long long)gridDim.x * ROWS, last = P.rows - 1;
    // operand o (0: dy, 1: h, 2: dh) of this thread's row in a stage
    auto room = [&](int stage, int o) { return nb_ring + ((stage * 3 + o) * ROWS + sub) * R::ROOM; };
    auto copy = [&](int stage, int o, const T *base, long long ld, long long row) {
        if constexpr (A == 1) {
            constexpr int V = 16 / (int)sizeof(T);
#pragma unroll
            for (int i = 0; i < NV * 8 / V; ++i) {
                const int piece = i * TPR + t;
                copy_piece(room(stage, o) + piece * 16, base, row * ld, last * ld + P.cols, piece, P.cols);
            }
            if (t == 0) copy_piece(room(stage, o) + NV * 8 / V * TPR * 16, base, row * ld, last * ld + P.cols, NV * 8 / V * TPR, P.cols);
        } else {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * TPR + t) * 8;
                copy8<A>((u32)__cvta_generic_to_shared(room(stage, o) + c * (int)sizeof(T)), base + row * ld, c, P.cols);
            }
        }
    };
    auto ask = [&](long long row, int stage) {
        if (row < P.rows) {
            copy(stage, 0, (const T *)P.dy, P.ldy, row);
            copy(stage, 1, (const T *)P.h, P.ldh, row);
            if (P.dh) copy(stage, 2, (const T *)P.dh, P.ldd, row);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    float rstd_next = 0.0f, rstd_last = 0.0f;
    auto rstd_at = [&](long long row) { return row < P.rows ? P.rstd[row] : 0.0f; };
#pragma unroll
    for (int i = 0; i < S - 1; ++i) ask(first + i * step, i);
    rstd_next = rstd_at(first);
    if (S == 3) rstd_last = rstd_at(first + step);
    int phase = 0, stage = 0;
    for (long long row = first; row < P.rows; row += step, phase ^= 1) {
        const float rstd = rstd_next;
        rstd_next = S == 3 ? rstd_last : rstd_at(row + step);
        if (S == 3) rstd_last = rstd_at(row + 2 * step);
        // the row is here; where its threads share their copies they meet, which also says that the stage before has been read
        asm volatile("cp.async.wait_group %0;" :: "n"(S - 2) : "memory");
        if constexpr (A == 1) {
            if (TPR == 32) __syncwarp();
            else __syncthreads();
        }
        ask(row + (S - 1) * step, stage == 0 ? S - 1 : stage - 1);
        auto take = [&](int o, int v, const void *base, long long ld) {
            const int c = (v * TPR + t) * 8;
            if constexpr (A == 1) return from_pieces<T>(room(stage, o), begins_by((const T *)base + row * ld), c, P.cols);
            else return *reinterpret_cast<const Eight<T> *>(room(stage, o) + c * (int)sizeof(T));
        };
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (!KEEP) load_gain<T, A>(P.gain, P.gain_f32, (v * TPR + t) * 8, P.cols, g[v]);
            float dy[8], h[8];
            widen(take(0, v, P.dy, P.ldy), dy);
            widen(take(1, v, P.h, P.ldh), h);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p = dy[i] * (h[i] * rstd);
                acc[v][i] += p;
                sum = fmaf(p, g[v][i], sum);
            }
        }
        if (P.dx || P.codes) {                          // (the same for all)
            const float q = row_sum<TPR>(sum, slots[phase]) * P.inv_cols;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (!KEEP) load_gain<T, A>(P.gain, P.gain_f32, (v * TPR + t) * 8, P.cols, g[v]);
                Eight<T> dy = take(0, v, P.dy, P.ldy), h = take(1, v, P.h, P.ldh), dh;
                if (P.dh) dh = take(2, v, P.dh, P.ldd);
                hold(dy);
                hold(h);
                norm_back_out<T, A>(P, row, (v * TPR + t) * 8, dy, h, dh, g[v], rstd, q, turn);
            }
        }
        stage = stage + 1 == S ? 0 : stage + 1;
    }
    if (!P.part) return;
    float *part = P.part + ((long long)blockIdx.x * ROWS + sub) * P.ld_part;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * TPR + t) * 8;
        if (c >= P.ld_part) continue;                   // (ld_part is a multiple of 8)
        *reinterpret_cast<float4 *>(part + c) = make_float4(acc[v][0], acc[v][1], acc[v][2], acc[v][3]);
        *reinterpret_cast<float4 *>(part + c + 4) = make_float4(acc[v][4], acc[v][5], acc[v][6], acc[v][7]);
    }
}

// Longer rows: dx by a CTA per row that reads it twice ...
template <class T, int A, int TPR>
__global__ void __launch_bounds__(TPR) k_norm_backward_long(const __grid_constant__ NormBackParams P)
{
    __shared__ float slots[32];
    __shared__ Eight<T> s_turns[Turns<A, T, TPR>::N];
    Eight<T> *turn = s_turns + (A == 1 ? threadIdx.x / 32 * 32 : 0);
    pdl_wait();
    pdl_launch_dependents();
    const long long row = blockIdx.x;
    const T *dyr = (const T *)P.dy + row * P.ldy, *hr = (const T *)P.h + row * P.ldh;
    const float rstd = P.rstd[row];
    float sum = 0.0f, g[8];
    for (int c = threadIdx.x * 8; c < P.cols; c += TPR * 8) {
        const Eight<T> dy = load8<A>(dyr, c, P.cols), h = load8<A>(hr, c, P.cols);
        load_gain<T, A>(P.gain, P.gain_f32, c, P.cols, g);
        float part = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) part = fmaf(dy[i] * (h[i] * rstd), g[i], part);
        sum += part;
    }
    const float q = row_sum<TPR>(sum, slots) * P.inv_cols;
    for (int c0 = 0; c0 < P.cols; c0 += TPR * 8) {
        const int c = c0 + threadIdx.x * 8;
        const Eight<T> dy = load8<A>(dyr, c, P.cols), h = load8<A>(hr, c, P.cols);
        Eight<T> dh;
        if (P.dh) dh = load8<A>((const T *)P.dh + row * P.ldd, c, P.cols);
        load_gain<T, A>(P.gain, P.gain_f32, c, P.cols, g);
        norm_back_out<T, A>(P, row, c, dy, h, dh, g, rstd, q, turn);
    }
}

// ... and the sums for dgain by strips of THREADS * 8 columns, ahead of it (dx may be dy itself): a CTA takes every
// gridDim.y-th row.
template <class T, int A>
__global__ void __launch_bounds__(THREADS) k_norm_dgain_long(const __grid_constant__ NormBackParams P)
{
    pdl_wait();
    pdl_launch_dependents();
    const int c = (int)(blockIdx.x * THREADS + threadIdx.x) * 8;
    if (c >= P.ld_part) return;
    float acc[8] = {};
    for (long long row = blockIdx.y; row < P.rows; row += gridDim.y) {
        const Eight<T> dy = load8<A>((const T *)P.dy + row * P.ldy, c, P.cols), h = load8<A>((const T *)P.h + row * P.ldh, c, P.cols);
        const float rstd = P.rstd[row];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += dy[i] * (h[i] * rstd);
    }
    float *part = P.part + (long long)blockIdx.y * P.ld_part + c;
    *reinterpret_cast<float4 *>(part) = make_float4(acc[0], acc[1], acc[2], acc[3]);
    *reinterpret_cast<float4 *>(part + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
}

// dgain = (dgain +) the sum of the slots: a CTA takes 32 columns, a warp every 32nd slot, the warps' sums are added in order.
constexpr int DGAIN_WARPS = 32;
static __global__ void __launch_bounds__(DGAIN_WARPS * 32) k_norm_dgain(const float *part, long long ld, int slots, float *dgain, int cols, int accumulate)
{
    __shared__ float s[DGAIN_WARPS][33];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = (int)blockIdx.x * 32 + lane;
    float sum = 0.0f;
    if (c < cols) {
#pragma unroll 8
        for (int i = warp; i < slots; i += DGAIN_WARPS) sum += part[i * ld + c];
    }
    s[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && c < cols) {
#pragma unroll
        for (int i = 1; i < DGAIN_WARPS; ++i) sum += s[i][lane];
        dgain[c] = accumulate ? dgain[c] + sum : sum;
    }
}

// ------------------------------------------------------------------ encoders
struct EncodeParams {
    const void *x;
    u8 *codes, *scales;
    float *theta;                       // blocks: the values that the codes stand for; NULL: not written
    long long ldx, ldc, lds, ld_theta;
    long long rows;
    int cols;
    u32 groups;                         // of a row
    u32 runs, reciprocal;               // rows: runs of groups of a row; floor(2^32 / runs), at most 2^32 - 1
};

// Largest magnitude of eight values as they lie in memory; no number if one of them is none. Patterns of 16-bit values
// are compared two at a time.
__device__ __forceinline__ float most_raw(const Eight<float> &e)
{
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = e.v[i];
    return most_of(v);
}
template <class T>
__device__ __forceinline__ float most_raw(const Eight<T> &e)
{
    const uint4 w = *reinterpret_cast<const uint4 *>(&e);
    constexpr u32 M = 0x7FFF7FFFu;
    const u32 m = __vimax3_s16x2(__vimax3_s16x2(w.x & M, w.y & M, w.z & M), w.w & M, 0);
    const u16 top = (u16)max(m & 0xFFFFu, m >> 16);
    return to_f32(*reinterpret_cast<const T *>(&top));
}

// Rows: nothing is shared between groups, so half-warps take them one after the other, whatever rows they lie in: runs of NG
// neighbouring groups of a row, for which a place is found once (8192 x 6000 in bf16: 26.3 us, 22.6 for the bytes; with a place for
// each group 28.5).
template <class T, int A, int NG>
__global__ void __launch_bounds__(THREADS) k_encode_rows(const __grid_constant__ EncodeParams P)
{
    pdl_wait();
    pdl_launch_dependents();
    constexpr int HALVES = THREADS / GROUP_LANES, UNITS = ENC_UNITS / NG;
    const int half = threadIdx.x / GROUP_LANES, lane = threadIdx.x % GROUP_LANES;
    const u32 units = (u32)P.rows * P.runs, first = blockIdx.x * (HALVES * UNITS) + half;
    u32 row[UNITS];
    int c[UNITS];
    Asked<A, T> asked[UNITS][NG];
    const long long total = (P.rows - 1) * P.ldx + P.cols;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        const u32 u = first + i * HALVES;
        u32 g;
        place_of_run(u, P.runs, P.reciprocal, [](u32 a, u32 b) { return __umulhi(a, b); }, row[i], g);
        c[i] = u < units ? (int)g * (NG * GROUP) + lane * 8 : P.cols;    // (P.cols: nothing to read or write)
#pragma unroll
        for (int k = 0; k < NG; ++k) asked[i][k] = ask8<A>((const T *)P.x, row[i] * P.ldx, total, c[i] + k * GROUP, P.cols);
    }
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        u8 *codes = P.codes + row[i] * P.ldc, *scales = P.scales + row[i] * P.lds;
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            const int at = c[i] + k * GROUP;
            const Eight<T> e = take8<A>(asked[i][k], (const T *)P.x, row[i] * P.ldx, at, P.cols);
            float v[8];
            widen(e, v);
            float most = group_most(most_raw(e), 0xFFFFFFFFu);
            if (is_odd(most)) {
                most = group_most(most_finite(v), 0xFFFFu << (threadIdx.x & 16));
                odd_to_nan(v);
            }
            const u32 s = scale_of(most);
            if (at < P.cols) {
                store_codes<A>(codes, at, P.cols, codes_of(v, scale_inverse(s)));
                if (lane == 0) scales[(u32)at / GROUP] = (u8)s;
            }
        }
    }
}

// Blocks of 128 x 128: a CTA each, thirty-two rows at a time. Measured: 33278 x 1500 bf16 29 us (23 for the bytes), 6000 x 1500 fp32 with theta
// 19 us (12).
constexpr int ENC_BLOCK = 512;
template <class T, int A>
__global__ void __launch_bounds__(ENC_BLOCK) k_encode_blocks(const __grid_constant__ EncodeParams P)
{
    constexpr int STEP = ENC_BLOCK / GROUP_LANES, N = GROUP / STEP, W = ENC_BLOCK / 32;
    __shared__ float s_most[2][W];
    __shared__ Eight<float> s_turns[Turns<A, float, ENC_BLOCK>::N];
    pdl_wait();
    pdl_launch_dependents();
    const u32 bi = blockIdx.x / P.groups, bj = blockIdx.x - bi * P.groups;
    const int c = (int)bj * GROUP + threadIdx.x % GROUP_LANES * 8;
    const long long r0 = (long long)bi * GROUP + threadIdx.x / GROUP_LANES;
    Asked<A, T> asked[N];
    const long long total = (P.rows - 1) * P.ldx + P.cols;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const long long r = r0 + i * STEP;
        asked[i] = ask8<A>((const T *)P.x, r * P.ldx, total, r < P.rows ? c : P.cols, P.cols);
    }
    Eight<T> e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = take8<A>(asked[i], (const T *)P.x, (r0 + i * STEP) * P.ldx, c, P.cols);
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) most = most2(most, most_raw(e[i]));
    auto join = [&](float *slot) {      // over the CTA
        most = group_most(most, 0xFFFFFFFFu);
        most = most2(most, __shfl_xor_sync(0xFFFFFFFFu, most, 16));
        if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = most;
        __syncthreads();
        const float x = slot[threadIdx.x % W];
        most = group_most(x, 0xFFFFFFFFu);
    };
    static_assert(W == GROUP_LANES, "the warps' maxima are one per lane of a group");
    join(s_most[0]);
    const bool odd = is_odd(most);      // (the same for the CTA)
    if (odd) {
        most = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float v[8];
            widen(e[i], v);
            most = fmaxf(most, most_finite(v));
        }
        join(s_most[1]);
    }
    const u32 s = scale_of(most);
    const float inverse = scale_inverse(s), scale = scale_value(s);
    if (threadIdx.x == 0) P.scales[bi * P.lds + bj] = (u8)s;
    const int lane = threadIdx.x % GROUP_LANES;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const long long r = r0 + i * STEP;
        if (A != 1 && (r >= P.rows || c >= P.cols)) continue;
        float v[8];
        widen(e[i], v);
        if (odd) odd_to_nan(v);
        const uint2 q = codes_of(v, inverse);
        const bool there = A != 1 || (r < P.rows && c < P.cols);
        if (there) store_codes<A>(P.codes + r * P.ldc, c, P.cols, q);
        if (!P.theta) continue;
        Eight<float> o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32 h2;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((u16)((j < 2 ? q.x : q.y) >> (16 * (j & 1)))));
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h2));
            o.v[2 * j] = f.x * scale;
            o.v[2 * j + 1] = f.y * scale;
        }
        float *row = P.theta + r * P.ld_theta;
        if constexpr (A != 1) {
            if (there) store8<A>(row, c, P.cols, o);
        } else {                        // through shared memory and out 16 neighbours at a time (whole warps are here)
            float *turn = reinterpret_cast<float *>(s_turns + threadIdx.x / GROUP_LANES * GROUP_LANES);
            __syncwarp();
            reinterpret_cast<Eight<float> *>(turn)[lane] = o;
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int at = (int)bj * GROUP + j * GROUP_LANES + lane;
                if (r < P.rows && at < P.cols) row[at] = turn[j * GROUP_LANES + lane];
            }
        }
    }
}

}  // namespace cs
