// Root-mean-square norm of rows with the residual's addition, forward and backward, and the encoders of rows and of blocks.
//
// All of it is bound by memory: a few operations for every 2 to 16 bytes. So each value is read once and kept, as it came, in
// the registers of the threads that share a row (TPR of them, NV times eight neighbouring columns each) while the row's sum
// is formed, and everything that is written leaves in the same pass, codes and scales included: a group of 128 columns
// is 16 neighbouring lanes, its largest magnitude four shuffles.
#pragma once
#include "coded.cuh"

namespace cs {

struct NormParams {
    const void *x, *residual, *gain;
    void *h, *y;
    u8 *codes, *scales;
    float *rstd;
    long long ldx, ldr, ldh, ldy, ldc, lds;
    long long rows;
    int cols;
    int vx, vr, vh, vy, vg;             // accesses that the rows allow
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
    int vy, vd, vh, vx, vg;
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

__device__ __forceinline__ float rstd_of(float sum, int cols, float eps) { return 1.0f / sqrtf(sum / (float)cols + eps); }
__device__ __forceinline__ float rstd_of(double sum, int cols, float eps) { return (float)(1.0 / sqrt(sum / cols + (double)eps)); }

template <class T>
__device__ __forceinline__ void load_gain(const void *gain, int f32, int vec, long long c, int cols, float (&g)[8])
{
    if (!gain) {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = 1.0f;
    } else if (f32) {
        const Eight<float> e = load8((const float *)gain, c, cols, vec);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = e[i];
    } else {
        const Eight<T> e = load8((const T *)gain, c, cols, vec);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = e[i];
    }
}

// h of columns c .. c+7: x, or the rounded sum of x and the residual.
template <class T>
__device__ __forceinline__ Eight<T> load_h(const NormParams &P, long long row, long long c)
{
    Eight<T> h = load8((const T *)P.x + row * P.ldx, c, P.cols, P.vx);
    if (P.residual) {
        const Eight<T> r = load8((const T *)P.residual + row * P.ldr, c, P.cols, P.vr);
#pragma unroll
        for (int i = 0; i < 8; ++i) h.v[i] = from_f32<T>(h[i] + r[i]);
    }
    return h;
}

// What follows from eight values of h.
template <class T>
__device__ __forceinline__ void norm_out(const NormParams &P, long long row, long long c, const Eight<T> &h, float rstd)
{
    float g[8], y[8];
    load_gain<T>(P.gain, P.gain_f32, P.vg, c, P.cols, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = h[i] * rstd * g[i];
    if (P.y) {
        Eight<T> o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.v[i] = from_f32<T>(y[i]);
        store8((T *)P.y + row * P.ldy, c, P.cols, P.vy, o);
    }
    if (P.codes) {
        if (c + 8 > P.cols) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = c + i < P.cols ? y[i] : 0.0f;        // (a row that is no number)
        }
        encode8(y, P.codes + row * P.ldc, P.scales + row * P.lds, c, P.cols);
    }
}

template <int TPR> struct RowThreads {
    static constexpr int BLOCK = TPR < 128 ? 128 : TPR, ROWS = BLOCK / TPR;
};

template <class T, int TPR, int NV>
__global__ void __launch_bounds__(RowThreads<TPR>::BLOCK) k_norm_forward(const __grid_constant__ NormParams P)
{
    __shared__ float slots[32];
    __shared__ double wide[32];
    pdl_wait();
    pdl_launch_dependents();
    const long long row = (long long)blockIdx.x * RowThreads<TPR>::ROWS + threadIdx.x / TPR;
    if (row >= P.rows) return;                          // (whole rows of threads: no barrier misses them)
    const int t = threadIdx.x % TPR;
    Eight<T> h[NV];
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) h[v] = load_h<T>(P, row, (long long)(v * TPR + t) * 8);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if (P.h) store8((T *)P.h + row * P.ldh, (long long)(v * TPR + t) * 8, P.cols, P.vh, h[v]);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(h[v][i], h[v][i], sum);
    }
    sum = row_sum<TPR>(sum, slots);
    float rstd = rstd_of(sum, P.cols, P.eps);
    if (!(sum <= 3.4e38f)) {                            // beyond fp32, or not a number (the same for the row)
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
    for (int v = 0; v < NV; ++v) norm_out<T>(P, row, (long long)(v * TPR + t) * 8, h[v], rstd);
}

// Rows that are longer than the threads' registers: read twice, the second time mostly from L2.
template <class T, int TPR>
__global__ void __launch_bounds__(TPR) k_norm_forward_long(const __grid_constant__ NormParams P)
{
    __shared__ double slots[32];
    pdl_wait();
    pdl_launch_dependents();
    const long long row = blockIdx.x;
    double sum = 0.0;
    for (long long c = threadIdx.x * 8; c < P.cols; c += TPR * 8) {
        const Eight<T> h = load_h<T>(P, row, c);
        if (P.h) store8((T *)P.h + row * P.ldh, c, P.cols, P.vh, h);
        double part = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) part += (double)h[i] * h[i];
        sum += part;
    }
    const float rstd = rstd_of(row_sum<TPR>(sum, slots), P.cols, P.eps);
    if (threadIdx.x == 0 && P.rstd) P.rstd[row] = rstd;
    if (!P.y && !P.codes) return;
    for (long long c0 = 0; c0 < P.cols; c0 += TPR * 8) {            // (all lanes stay for the shuffles)
        const long long c = c0 + threadIdx.x * 8;
        // what this thread wrote to h, or x and the residual again where there is no h
        const Eight<T> h = P.h ? load8((const T *)P.h + row * P.ldh, c, P.cols, P.vh) : load_h<T>(P, row, c);
        norm_out<T>(P, row, c, h, rstd);
    }
}

// ------------------------------------------------------------------ backward
// dx of columns c .. c+7; q: the mean that is taken out.
template <class T>
__device__ __forceinline__ void norm_back_out(const NormBackParams &P, long long row, long long c, const Eight<T> &dy, const Eight<T> &h,
                                              const Eight<T> &dh, const float (&g)[8], float rstd, float q)
{
    float d[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        d[i] = rstd * fmaf(-(h[i] * rstd), q, dy[i] * g[i]);
        if (P.dh) d[i] += dh[i];
    }
    if (P.dx) {
        Eight<T> o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.v[i] = from_f32<T>(d[i]);
        store8((T *)P.dx + row * P.ldx, c, P.cols, P.vx, o);
    }
    if (P.codes) {
        if (c + 8 > P.cols) {
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = c + i < P.cols ? d[i] : 0.0f;
        }
        encode8(d, P.codes + row * P.ldc, P.scales + row * P.lds, c, P.cols);
    }
}

// A CTA takes every gridDim-th row (group of rows), so that a thread's sums for dgain stay in its registers; they leave
// once, as one of the slots that k_norm_dgain adds up.
template <class T, int TPR, int NV>
__global__ void __launch_bounds__(RowThreads<TPR>::BLOCK) k_norm_backward(const __grid_constant__ NormBackParams P)
{
    constexpr int ROWS = RowThreads<TPR>::ROWS;
    __shared__ float slots[2][32];
    pdl_wait();
    pdl_launch_dependents();
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    constexpr bool KEEP = TPR < 1024;                   // (a thread of 1024 has 64 registers: the gain is read again, from L1)
    float g[NV][8], acc[NV][8] = {};
#pragma unroll
    for (int v = 0; v < NV; ++v)
        if (KEEP) load_gain<T>(P.gain, P.gain_f32, P.vg, (long long)(v * TPR + t) * 8, P.cols, g[v]);
    int turn = 0;
    for (long long row = (long long)blockIdx.x * ROWS + sub; row < P.rows; row += (long long)gridDim.x * ROWS, turn ^= 1) {
        Eight<T> dy[NV], h[NV], dh[NV];
        const float rstd = P.rstd[row];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const long long c = (long long)(v * TPR + t) * 8;
            dy[v] = load8((const T *)P.dy + row * P.ldy, c, P.cols, P.vy);
            h[v] = load8((const T *)P.h + row * P.ldh, c, P.cols, P.vh);
            if (P.dh) dh[v] = load8((const T *)P.dh + row * P.ldd, c, P.cols, P.vd);
        }
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (!KEEP) load_gain<T>(P.gain, P.gain_f32, P.vg, (long long)(v * TPR + t) * 8, P.cols, g[v]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p = dy[v][i] * (h[v][i] * rstd);
                acc[v][i] += p;
                sum = fmaf(p, g[v][i], sum);
            }
        }
        if (!P.dx && !P.codes) continue;                // (the same for all)
        const float q = row_sum<TPR>(sum, slots[turn]) / (float)P.cols;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (!KEEP) load_gain<T>(P.gain, P.gain_f32, P.vg, (long long)(v * TPR + t) * 8, P.cols, g[v]);
            norm_back_out<T>(P, row, (long long)(v * TPR + t) * 8, dy[v], h[v], dh[v], g[v], rstd, q);
        }
    }
    if (!P.part) return;
    float *part = P.part + ((long long)blockIdx.x * ROWS + sub) * P.ld_part;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const long long c = (long long)(v * TPR + t) * 8;
        if (c >= P.ld_part) continue;                   // (ld_part is a multiple of 8)
        *reinterpret_cast<float4 *>(part + c) = make_float4(acc[v][0], acc[v][1], acc[v][2], acc[v][3]);
        *reinterpret_cast<float4 *>(part + c + 4) = make_float4(acc[v][4], acc[v][5], acc[v][6], acc[v][7]);
    }
}

// Longer rows: dx by a CTA per row that reads it twice ...
template <class T, int TPR>
__global__ void __launch_bounds__(TPR) k_norm_backward_long(const __grid_constant__ NormBackParams P)
{
    __shared__ float slots[32];
    pdl_wait();
    pdl_launch_dependents();
    const long long row = blockIdx.x;
    const T *dyr = (const T *)P.dy + row * P.ldy, *hr = (const T *)P.h + row * P.ldh;
    const float rstd = P.rstd[row];
    float sum = 0.0f, g[8];
    for (long long c = threadIdx.x * 8; c < P.cols; c += TPR * 8) {
        const Eight<T> dy = load8(dyr, c, P.cols, P.vy), h = load8(hr, c, P.cols, P.vh);
        load_gain<T>(P.gain, P.gain_f32, P.vg, c, P.cols, g);
        float part = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) part = fmaf(dy[i] * (h[i] * rstd), g[i], part);
        sum += part;
    }
    const float q = row_sum<TPR>(sum, slots) / (float)P.cols;
    for (long long c0 = 0; c0 < P.cols; c0 += TPR * 8) {
        const long long c = c0 + threadIdx.x * 8;
        const Eight<T> dy = load8(dyr, c, P.cols, P.vy), h = load8(hr, c, P.cols, P.vh);
        Eight<T> dh;
        if (P.dh) dh = load8((const T *)P.dh + row * P.ldd, c, P.cols, P.vd);
        load_gain<T>(P.gain, P.gain_f32, P.vg, c, P.cols, g);
        norm_back_out<T>(P, row, c, dy, h, dh, g, rstd, q);
    }
}

// ... and the sums for dgain by strips of THREADS * 8 columns, ahead of it (dx may be dy itself): a CTA takes every
// gridDim.y-th row.
template <class T>
__global__ void __launch_bounds__(THREADS) k_norm_dgain_long(const __grid_constant__ NormBackParams P)
{
    pdl_wait();
    pdl_launch_dependents();
    const long long c = ((long long)blockIdx.x * THREADS + threadIdx.x) * 8;
    if (c >= P.ld_part) return;
    float acc[8] = {};
    for (long long row = blockIdx.y; row < P.rows; row += gridDim.y) {
        const Eight<T> dy = load8((const T *)P.dy + row * P.ldy, c, P.cols, P.vy), h = load8((const T *)P.h + row * P.ldh, c, P.cols, P.vh);
        const float rstd = P.rstd[row];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += dy[i] * (h[i] * rstd);
    }
    float *part = P.part + (long long)blockIdx.y * P.ld_part + c;
    *reinterpret_cast<float4 *>(part) = make_float4(acc[0], acc[1], acc[2], acc[3]);
    *reinterpret_cast<float4 *>(part + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
}

// dgain = (dgain +) the sum of the slots, in their order by eighths. A CTA takes 32 columns, a warp every eighth slot.
__global__ void __launch_bounds__(THREADS) k_norm_dgain(const float *part, long long ld, int slots, float *dgain, int cols, int accumulate)
{
    __shared__ float s[WARPS][32];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane;
    float sum = 0.0f;
    if (c < cols) {
#pragma unroll 8
        for (int i = warp; i < slots; i += WARPS) sum += part[i * ld + c];
    }
    s[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && c < cols) {
#pragma unroll
        for (int i = 1; i < WARPS; ++i) sum += s[i][lane];
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
    int groups;                         // of a row
    int vx, vt;
};

constexpr int ENC_UNITS = 4;            // groups of a half-warp, all of whose loads leave together

// Rows: nothing is shared between groups, so half-warps take them one after the other, whatever rows they lie in.
template <class T>
__global__ void __launch_bounds__(THREADS) k_encode_rows(const __grid_constant__ EncodeParams P)
{
    pdl_wait();
    pdl_launch_dependents();
    constexpr int HALVES = THREADS / GROUP_LANES;
    const int half = threadIdx.x / GROUP_LANES, lane = threadIdx.x % GROUP_LANES;
    const u64 units = (u64)P.rows * (u32)P.groups, first = (u64)blockIdx.x * (HALVES * ENC_UNITS);
    long long row[ENC_UNITS];
    int c[ENC_UNITS];
    Eight<T> e[ENC_UNITS];
#pragma unroll
    for (int i = 0; i < ENC_UNITS; ++i) {
        const u64 u = first + i * HALVES + half;
        const u64 r = units >> 32 ? u / (u32)P.groups : (u64)((u32)u / (u32)P.groups);
        const bool live = u < units;
        row[i] = live ? (long long)r : 0;
        c[i] = live ? (int)(u - r * (u32)P.groups) * GROUP + lane * 8 : P.cols;        // (P.cols: nothing to read or write)
        e[i] = load8((const T *)P.x + row[i] * P.ldx, c[i], P.cols, P.vx);
    }
#pragma unroll
    for (int i = 0; i < ENC_UNITS; ++i) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = e[i][j];
        encode8(v, P.codes + row[i] * P.ldc, P.scales + row[i] * P.lds, c[i], P.cols);
    }
}

// Blocks of 128 x 128: a CTA each, sixteen rows at a time.
template <class T>
__global__ void __launch_bounds__(THREADS) k_encode_blocks(const __grid_constant__ EncodeParams P)
{
    __shared__ u32 s_most[2][WARPS];
    pdl_wait();
    pdl_launch_dependents();
    constexpr int STEP = THREADS / GROUP_LANES, N = GROUP / STEP;
    const long long bj = blockIdx.x % P.groups, bi = blockIdx.x / P.groups;
    const long long c = bj * GROUP + threadIdx.x % GROUP_LANES * 8, r0 = bi * GROUP + threadIdx.x / GROUP_LANES;
    Eight<T> e[N];
    u32 most = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const long long r = r0 + i * STEP;
        e[i] = load8((const T *)P.x + min(r, P.rows - 1) * P.ldx, r < P.rows ? c : (long long)P.cols, P.cols, P.vx);
    }
    bool odd = false;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {              // a second time only where something is not finite
        most = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = e[i][j];
            most = max(most, most_of(v, pass == 1));
        }
        most = __reduce_max_sync(0xFFFFFFFFu, most);
        if ((threadIdx.x & 31) == 0) s_most[pass][threadIdx.x >> 5] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WARPS; ++w) most = max(most, s_most[pass][w]);
        if (most < 0x7F800000u) break;                  // (the same for the CTA)
        odd = true;
    }
    const u32 s = scale_of(most);
    const float inverse = scale_inverse(s), scale = scale_value(s);
    if (threadIdx.x == 0) P.scales[bi * P.lds + bj] = (u8)s;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const long long r = r0 + i * STEP;
        if (r >= P.rows || c >= P.cols) continue;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = e[i][j];
        const uint2 q = codes_of(v, inverse, odd);
        store_codes(P.codes + r * P.ldc, c, P.cols, q);
        if (P.theta) {
            Eight<float> o;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u32 h2;
                asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((u16)((j < 2 ? q.x : q.y) >> (16 * (j & 1)))));
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h2));
                o.v[2 * j] = f.x * scale;
                o.v[2 * j + 1] = f.y * scale;
            }
            store8(P.theta + r * P.ld_theta, c, P.cols, P.vt, o);
        }
    }
}

}  // namespace cs
