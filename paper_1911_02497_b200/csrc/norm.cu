// Host side of the norm and of the encoders: argument checks, launches.
#include <cmath>
#include <new>

#include "norm.cuh"
#include "op_args.h"

using namespace cs;

static_assert(CONDENSA_CODE_GROUP == GROUP, "columns that share a scale");

namespace {

// CTAs of a kernel that an SM holds.
int resident_ctas(condensa_ctx *ctx, const void *f, int block, int &count)
{
    for (const condensa_ctx::ClusterFit &k : ctx->cluster_fit)
        if (k.f == f && k.size == 0) {
            count = k.count;
            return CONDENSA_OK;
        }
    count = 0;
    CU_TRY(ctx, cudaOccupancyMaxActiveBlocksPerMultiprocessor(&count, f, block, 0));
    if (count < 1) count = 1;
    ctx->cluster_fit.push_back({f, 0, count});
    return CONDENSA_OK;
}

constexpr int LONG_TPR = 512;           // threads of a row that is read twice

// ------------------------------------------------------------------ forward
template <class T, int TPR, int NV>
int forward_as(condensa_ctx *ctx, const NormParams &P, cudaStream_t stream)
{
    constexpr int ROWS = RowThreads<TPR>::ROWS;
    return op_launch(ctx, "k_norm_forward", k_norm_forward<T, TPR, NV>, dim3((unsigned)((P.rows + ROWS - 1) / ROWS)), RowThreads<TPR>::BLOCK, stream, P);
}

// The threads of a row: as many as hold it with one or two eights each.
template <class T>
int forward_of(condensa_ctx *ctx, const NormParams &P, cudaStream_t stream)
{
    const int eights = (P.cols + 7) / 8;
    return eights <= 32   ? forward_as<T, 32, 1>(ctx, P, stream)
         : eights <= 64   ? forward_as<T, 32, 2>(ctx, P, stream)
         : eights <= 128  ? forward_as<T, 128, 1>(ctx, P, stream)
         : eights <= 256  ? forward_as<T, 128, 2>(ctx, P, stream)
         : eights <= 512  ? forward_as<T, 256, 2>(ctx, P, stream)
         : eights <= 1024 ? forward_as<T, 512, 2>(ctx, P, stream)
         : eights <= 2048 ? forward_as<T, 1024, 2>(ctx, P, stream)
                          : op_launch(ctx, "k_norm_forward_long", k_norm_forward_long<T, LONG_TPR>, dim3((unsigned)P.rows), LONG_TPR, stream, P);
}

int forward(condensa_ctx *ctx, const condensa_norm *p, cudaStream_t stream)
{
    if (!p) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "norm is NULL");
    if (!op_known_type(p->dtype)) return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "dtype must be CONDENSA_DTYPE_FP32, _FP16 or _BF16");
    if (p->gain && p->gain_dtype != CONDENSA_DTYPE_FP32 && p->gain_dtype != p->dtype)
        return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "gain_dtype must be CONDENSA_DTYPE_FP32 or dtype");
    if (p->reserved) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "reserved must be 0");
    if (!(p->eps > 0.0f) || !std::isfinite(p->eps)) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "eps must be positive and finite");
    OpArgs a{ctx};
    int rc = a.sizes(p->rows, p->cols);
    if (rc || p->rows == 0) return rc;
    const int e = op_type_bytes(p->dtype), ge = op_type_bytes(p->gain_dtype);
    if ((uintptr_t)p->gain % ge || (uintptr_t)p->rstd % 4) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "gain or rstd is not aligned to its type");
    const bool coded = p->code.codes != nullptr;
    if (p->h && (rc = a.matrix("h", p->h, p->ldh, p->rows, p->cols, e, true)) != 0) return rc;
    if (p->y && (rc = a.matrix("y", p->y, p->ldy, p->rows, p->cols, e, true)) != 0) return rc;
    if (coded && (rc = a.coded("code", p->code, p->rows, p->cols, 1, true)) != 0) return rc;
    // (an output may be an input itself; then the input is checked, but not noted a second time)
    auto input = [&](const char *name, const void *q, long long ld) {
        const bool itself = (q == p->h && ld == p->ldh) || (q == p->y && ld == p->ldy);
        const int r = a.matrix(name, q, ld, p->rows, p->cols, e, false);
        if (!r && itself) a.rows.pop_back();
        return r;
    };
    if ((rc = input("x", p->x, p->ldx)) != 0) return rc;
    if (p->residual && (rc = input("residual", p->residual, p->ld_residual)) != 0) return rc;
    a.array(p->gain, p->cols * ge, false);
    a.array(p->rstd, p->rows * 4, true);
    if ((rc = a.apart()) != 0) return rc;
    if (!p->h && !p->y && !coded && !p->rstd) return CONDENSA_OK;
    CU_TRY(ctx, cudaSetDevice(ctx->device));
    NormParams P;
    memset(&P, 0, sizeof(P));
    P.x = p->x; P.residual = p->residual; P.gain = p->gain;
    P.h = p->h; P.y = p->y; P.rstd = p->rstd;
    P.ldx = p->ldx; P.ldr = p->ld_residual; P.ldh = p->ldh; P.ldy = p->ldy;
    if (coded) {
        P.codes = p->code.codes; P.scales = p->code.scales;
        P.ldc = p->code.ld; P.lds = p->code.ld_scales;
    }
    P.rows = p->rows;
    P.cols = (int)p->cols;
    P.eps = p->eps;
    P.gain_f32 = p->gain_dtype == CONDENSA_DTYPE_FP32;
    P.vx = op_access(P.x, P.ldx, e);
    P.vr = op_access(P.residual, P.ldr, e);
    P.vh = op_access(P.h, P.ldh, e);
    P.vy = op_access(P.y, P.ldy, e);
    P.vg = op_access(P.gain, 0, ge);
    return p->dtype == CONDENSA_DTYPE_BF16 ? forward_of<__nv_bfloat16>(ctx, P, stream)
         : p->dtype == CONDENSA_DTYPE_FP16 ? forward_of<__half>(ctx, P, stream) : forward_of<float>(ctx, P, stream);
}

// ------------------------------------------------------------------ backward
// How a backward call is cut: CTAs, and the slots of sums for dgain that they leave.
struct BackPlan {
    int grid, slots;
};

template <class T, int TPR, int NV>
int backward_as(condensa_ctx *ctx, NormBackParams &P, BackPlan &plan, bool run, cudaStream_t stream)
{
    constexpr int ROWS = RowThreads<TPR>::ROWS, BLOCK = RowThreads<TPR>::BLOCK;
    auto k = k_norm_backward<T, TPR, NV>;
    if (run) return op_launch(ctx, "k_norm_backward", k, dim3((unsigned)plan.grid), BLOCK, stream, P);
    int fit = 1;
    const int rc = resident_ctas(ctx, (const void *)k, BLOCK, fit);
    if (rc) return rc;
    plan.grid = stream_grid(ctx, (P.rows + ROWS - 1) / ROWS, fit);
    plan.slots = plan.grid * ROWS;
    return CONDENSA_OK;
}

// The register file holds 64 values a thread of 1024, too few for fp32 operands.
template <class T> int longest_back() { return sizeof(T) == 4 ? 1024 : 2048; }

template <class T>
int backward_of(condensa_ctx *ctx, NormBackParams &P, BackPlan &plan, bool run, cudaStream_t stream)
{
    const int eights = (P.cols + 7) / 8;
    if (eights > longest_back<T>()) {
        const unsigned strips = (unsigned)((eights + THREADS - 1) / THREADS);
        if (!run) {
            plan.grid = stream_grid(ctx, P.rows, std::max(1, 4 / (int)strips));
            plan.slots = plan.grid;
            return CONDENSA_OK;
        }
        int rc = CONDENSA_OK;
        if (P.part) rc = op_launch(ctx, "k_norm_dgain_long", k_norm_dgain_long<T>, dim3(strips, (unsigned)plan.grid), THREADS, stream, P);
        if (rc || (!P.dx && !P.codes)) return rc;
        return op_launch(ctx, "k_norm_backward_long", k_norm_backward_long<T, LONG_TPR>, dim3((unsigned)P.rows), LONG_TPR, stream, P);
    }
    if constexpr (sizeof(T) == 2)
        if (eights > 1024) return backward_as<T, 1024, 2>(ctx, P, plan, run, stream);
    return eights <= 32  ? backward_as<T, 32, 1>(ctx, P, plan, run, stream)
         : eights <= 64  ? backward_as<T, 32, 2>(ctx, P, plan, run, stream)
         : eights <= 128 ? backward_as<T, 128, 1>(ctx, P, plan, run, stream)
         : eights <= 256 ? backward_as<T, 128, 2>(ctx, P, plan, run, stream)
         : eights <= 512 ? backward_as<T, 256, 2>(ctx, P, plan, run, stream)
                         : backward_as<T, 512, 2>(ctx, P, plan, run, stream);
}

int backward_type(condensa_ctx *ctx, int dtype, NormBackParams &P, BackPlan &plan, bool run, cudaStream_t stream)
{
    return dtype == CONDENSA_DTYPE_BF16 ? backward_of<__nv_bfloat16>(ctx, P, plan, run, stream)
         : dtype == CONDENSA_DTYPE_FP16 ? backward_of<__half>(ctx, P, plan, run, stream) : backward_of<float>(ctx, P, plan, run, stream);
}

int backward(condensa_ctx *ctx, const condensa_norm_gradient *p, cudaStream_t stream)
{
    if (!p) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "norm is NULL");
    if (!op_known_type(p->dtype)) return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "dtype must be CONDENSA_DTYPE_FP32, _FP16 or _BF16");
    if (p->gain && p->gain_dtype != CONDENSA_DTYPE_FP32 && p->gain_dtype != p->dtype)
        return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "gain_dtype must be CONDENSA_DTYPE_FP32 or dtype");
    if (p->reserved) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "reserved must be 0");
    OpArgs a{ctx};
    int rc = a.sizes(p->rows, p->cols);
    if (rc) return rc;
    const int e = op_type_bytes(p->dtype), ge = op_type_bytes(p->gain_dtype);
    if ((uintptr_t)p->gain % ge || (uintptr_t)p->rstd % 4 || (uintptr_t)p->dgain % 4)
        return fail(ctx, CONDENSA_ERR_INVALID_ARG, "gain, rstd or dgain is not aligned to its type");
    const bool coded = p->code.codes != nullptr;
    if (p->rows > 0) {
        if (!p->rstd) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "rstd is NULL");
        if (p->dx && (rc = a.matrix("dx", p->dx, p->ld_dx, p->rows, p->cols, e, true)) != 0) return rc;
        if (coded && (rc = a.coded("code", p->code, p->rows, p->cols, 1, true)) != 0) return rc;
        auto input = [&](const char *name, const void *q, long long ld, bool may) {
            const bool itself = may && q == p->dx && ld == p->ld_dx;
            const int r = a.matrix(name, q, ld, p->rows, p->cols, e, false);
            if (!r && itself) a.rows.pop_back();
            return r;
        };
        if ((rc = input("dy", p->dy, p->ld_dy, true)) != 0) return rc;
        if ((rc = input("h", p->h, p->ldh, false)) != 0) return rc;
        if (p->dh && (rc = input("dh", p->dh, p->ld_dh, true)) != 0) return rc;
        a.array(p->rstd, p->rows * 4, false);
    }
    a.array(p->gain, p->cols * ge, false);
    a.array(p->dgain, p->cols * 4, true);
    if ((rc = a.apart()) != 0) return rc;
    if (p->rows == 0 && (!p->dgain || p->accumulate)) return CONDENSA_OK;
    if (!p->dx && !coded && !p->dgain) return CONDENSA_OK;
    CU_TRY(ctx, cudaSetDevice(ctx->device));
    NormBackParams P;
    memset(&P, 0, sizeof(P));
    P.dy = p->dy; P.dh = p->dh; P.h = p->h; P.gain = p->gain; P.rstd = p->rstd; P.dx = p->dx;
    P.ldy = p->ld_dy; P.ldd = p->ld_dh; P.ldh = p->ldh; P.ldx = p->ld_dx;
    if (coded) {
        P.codes = p->code.codes; P.scales = p->code.scales;
        P.ldc = p->code.ld; P.lds = p->code.ld_scales;
    }
    P.rows = p->rows;
    P.cols = (int)p->cols;
    P.gain_f32 = p->gain_dtype == CONDENSA_DTYPE_FP32;
    P.vy = op_access(P.dy, P.ldy, e);
    P.vd = op_access(P.dh, P.ldd, e);
    P.vh = op_access(P.h, P.ldh, e);
    P.vx = op_access(P.dx, P.ldx, e);
    P.vg = op_access(P.gain, 0, ge);
    P.ld_part = (P.cols + 7) / 8 * 8;
    BackPlan plan = {0, 0};
    OpWorkspaceUse use;
    if (p->rows > 0 && (rc = backward_type(ctx, p->dtype, P, plan, false, stream)) != 0) return rc;
    if (p->dgain && plan.slots) {
        if ((rc = op_workspace(ctx, 256 + sizeof(float) * (size_t)plan.slots * (size_t)P.ld_part, stream, use)) != 0) return rc;
        P.part = (float *)(ctx->op.p + 256);
    }
    if (p->rows > 0 && (rc = backward_type(ctx, p->dtype, P, plan, true, stream)) != 0) return rc;
    if (p->dgain) {
        rc = op_launch(ctx, "k_norm_dgain", k_norm_dgain, dim3((unsigned)((P.cols + 31) / 32)), THREADS, stream, (const float *)P.part, P.ld_part, plan.slots,
                       p->dgain, P.cols, p->accumulate ? 1 : 0);
        if (rc) return rc;
    }
    return op_workspace_done(ctx, use);
}

// ------------------------------------------------------------------ encoders
int encode_rows(condensa_ctx *ctx, const void *x, long long ldx, long long rows, long long cols, int dtype, const condensa_coded *out, cudaStream_t stream)
{
    if (!out) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "out is NULL");
    if (!op_known_type(dtype)) return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "dtype must be CONDENSA_DTYPE_FP32, _FP16 or _BF16");
    OpArgs a{ctx};
    int rc = a.sizes(rows, cols);
    if (rc || rows == 0) return rc;
    const int e = op_type_bytes(dtype);
    if ((rc = a.matrix("x", x, ldx, rows, cols, e, false)) != 0) return rc;
    if ((rc = a.coded("out", *out, rows, cols, 1, true)) != 0) return rc;
    if ((rc = a.apart()) != 0) return rc;
    EncodeParams P;
    memset(&P, 0, sizeof(P));
    P.x = x; P.ldx = ldx;
    P.codes = out->codes; P.scales = out->scales; P.ldc = out->ld; P.lds = out->ld_scales;
    P.rows = rows;
    P.cols = (int)cols;
    P.groups = (int)((cols + GROUP - 1) / GROUP);
    P.vx = op_access(x, ldx, e);
    const long long per = THREADS / GROUP_LANES * ENC_UNITS, grid = (rows * P.groups + per - 1) / per;
    if (grid > 0x7FFFFFFFll) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "too many groups for one launch");
    CU_TRY(ctx, cudaSetDevice(ctx->device));
    return op_launch(ctx, "k_encode_rows", dtype == CONDENSA_DTYPE_BF16 ? k_encode_rows<__nv_bfloat16> : dtype == CONDENSA_DTYPE_FP16 ? k_encode_rows<__half> : k_encode_rows<float>,
                     dim3((unsigned)grid), THREADS, stream, P);
}

int encode_blocks(condensa_ctx *ctx, const void *w, long long ldw, long long n, long long k, int dtype, const condensa_coded *out, float *theta, long long ld_theta,
                  cudaStream_t stream)
{
    if (!out) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "out is NULL");
    if (!op_known_type(dtype)) return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "dtype must be CONDENSA_DTYPE_FP32, _FP16 or _BF16");
    if (n < 1 || k < 1) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "n and k must be positive");
    if (n > OP_MAX_WIDTH || k > OP_MAX_WIDTH) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "n and k must not exceed 2^22");
    OpArgs a{ctx};
    const int e = op_type_bytes(dtype);
    int rc = a.matrix("w", w, ldw, n, k, e, false);
    if (rc) return rc;
    if (theta && (const void *)theta == w && ld_theta == ldw && e == 4) a.rows.pop_back();
    if (theta && (rc = a.matrix("theta", theta, ld_theta, n, k, 4, true)) != 0) return rc;
    if ((rc = a.coded("out", *out, n, k, GROUP, true)) != 0) return rc;
    if ((rc = a.apart()) != 0) return rc;
    EncodeParams P;
    memset(&P, 0, sizeof(P));
    P.x = w; P.ldx = ldw;
    P.codes = out->codes; P.scales = out->scales; P.ldc = out->ld; P.lds = out->ld_scales;
    P.theta = theta; P.ld_theta = ld_theta;
    P.rows = n;
    P.cols = (int)k;
    P.groups = (int)((k + GROUP - 1) / GROUP);
    P.vx = op_access(w, ldw, e);
    P.vt = op_access(theta, ld_theta, 4);
    CU_TRY(ctx, cudaSetDevice(ctx->device));
    return op_launch(ctx, "k_encode_blocks",
                     dtype == CONDENSA_DTYPE_BF16 ? k_encode_blocks<__nv_bfloat16> : dtype == CONDENSA_DTYPE_FP16 ? k_encode_blocks<__half> : k_encode_blocks<float>,
                     dim3((unsigned)((n + GROUP - 1) / GROUP * P.groups)), THREADS, stream, P);
}

}  // namespace

extern "C" {

int condensa_norm_forward(condensa_ctx *ctx, const condensa_norm *norm, void *stream)
{
    if (!ctx) return CONDENSA_ERR_INVALID_ARG;
    try {
        return forward(ctx, norm, (cudaStream_t)stream);
    } catch (const std::bad_alloc &) {
        return fail(ctx, CONDENSA_ERR_WORKSPACE, "out of host memory");
    }
}

int condensa_norm_backward(condensa_ctx *ctx, const condensa_norm_gradient *norm, void *stream)
{
    if (!ctx) return CONDENSA_ERR_INVALID_ARG;
    try {
        return backward(ctx, norm, (cudaStream_t)stream);
    } catch (const std::bad_alloc &) {
        return fail(ctx, CONDENSA_ERR_WORKSPACE, "out of host memory");
    }
}

int condensa_encode_rows(condensa_ctx *ctx, const void *x, int64_t ldx, int64_t rows, int64_t cols, int dtype, const condensa_coded *out, void *stream)
{
    if (!ctx) return CONDENSA_ERR_INVALID_ARG;
    try {
        return encode_rows(ctx, x, ldx, rows, cols, dtype, out, (cudaStream_t)stream);
    } catch (const std::bad_alloc &) {
        return fail(ctx, CONDENSA_ERR_WORKSPACE, "out of host memory");
    }
}

int condensa_encode_blocks(condensa_ctx *ctx, const void *w, int64_t ldw, int64_t n, int64_t k, int dtype, const condensa_coded *out, float *theta,
                           int64_t ld_theta, void *stream)
{
    if (!ctx) return CONDENSA_ERR_INVALID_ARG;
    try {
        return encode_blocks(ctx, w, ldw, n, k, dtype, out, theta, ld_theta, (cudaStream_t)stream);
    } catch (const std::bad_alloc &) {
        return fail(ctx, CONDENSA_ERR_WORKSPACE, "out of host memory");
    }
}

}  // extern "C"
