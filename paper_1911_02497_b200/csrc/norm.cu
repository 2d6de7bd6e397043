// Host side of the norm and of the encoders: argument checks, launches.
#include <cmath>
#include <new>

#include "norm_launch.cuh"

using namespace cs;

static_assert(CONDENSA_CODE_GROUP == GROUP, "columns that share a scale");

namespace {

// ------------------------------------------------------------------ forward
int forward(condensa_ctx *ctx, const condensa_norm *p, cudaStream_t stream)
{
    if (!p) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "norm is NULL");
    if (!op_known_type(p->dtype)) return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "dtype must be CONDENSA_DTYPE_FP32, _FP16 or _BF16");
    if (p->gain && p->gain_dtype != CONDENSA_DTYPE_FP32 && p->gain_dtype != p->dtype)
        return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "gain_dtype must be CONDENSA_DTYPE_FP32 or dtype");
    if (p->reserved) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "reserved must be 0");
    if (!(p->eps > 0.0f) || !std::isfinite(p->eps)) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "eps must be positive and finite");
    OpArgs a(ctx);
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
    P.inv_cols = 1.0f / (float)p->cols;
    P.eps = p->eps;
    P.gain_f32 = p->gain_dtype == CONDENSA_DTYPE_FP32;
    const int access = std::min({op_access(P.x, P.ldx, e, P.cols), op_access(P.residual, P.ldr, e, P.cols), op_access(P.h, P.ldh, e, P.cols),
                                 op_access(P.y, P.ldy, e, P.cols), op_access(P.gain, 0, ge, P.cols)});
    return p->dtype == CONDENSA_DTYPE_BF16 ? norm_forward_launch<__nv_bfloat16>(ctx, P, access, stream)
         : p->dtype == CONDENSA_DTYPE_FP16 ? norm_forward_launch<__half>(ctx, P, access, stream) : norm_forward_launch<float>(ctx, P, access, stream);
}

// ------------------------------------------------------------------ backward
int backward_type(condensa_ctx *ctx, int dtype, const NormBackParams &P, NormBackPlan &plan, int access, bool run, cudaStream_t stream)
{
    return dtype == CONDENSA_DTYPE_BF16 ? norm_backward_launch<__nv_bfloat16>(ctx, P, plan, access, run, stream)
         : dtype == CONDENSA_DTYPE_FP16 ? norm_backward_launch<__half>(ctx, P, plan, access, run, stream)
                                        : norm_backward_launch<float>(ctx, P, plan, access, run, stream);
}

int backward(condensa_ctx *ctx, const condensa_norm_gradient *p, cudaStream_t stream)
{
    if (!p) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "norm is NULL");
    if (!op_known_type(p->dtype)) return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "dtype must be CONDENSA_DTYPE_FP32, _FP16 or _BF16");
    if (p->gain && p->gain_dtype != CONDENSA_DTYPE_FP32 && p->gain_dtype != p->dtype)
        return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "gain_dtype must be CONDENSA_DTYPE_FP32 or dtype");
    if (p->reserved) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "reserved must be 0");
    OpArgs a(ctx);
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
    P.inv_cols = 1.0f / (float)p->cols;
    P.gain_f32 = p->gain_dtype == CONDENSA_DTYPE_FP32;
    const int access = std::min({op_access(P.dy, P.ldy, e, P.cols), op_access(P.dh, P.ldd, e, P.cols), op_access(P.h, P.ldh, e, P.cols),
                                 op_access(P.dx, P.ldx, e, P.cols), op_access(P.gain, 0, ge, P.cols)});
    P.ld_part = (P.cols + 7) / 8 * 8;
    NormBackPlan plan = {0, 0};
    OpWorkspaceUse use;
    if (p->rows > 0 && (rc = backward_type(ctx, p->dtype, P, plan, access, false, stream)) != 0) return rc;
    if (p->dgain && plan.slots) {
        if ((rc = op_workspace(ctx, 256 + sizeof(float) * (size_t)plan.slots * (size_t)P.ld_part, stream, use)) != 0) return rc;
        P.part = (float *)(ctx->op.p + 256);
    }
    if (p->rows > 0 && (rc = backward_type(ctx, p->dtype, P, plan, access, true, stream)) != 0) return rc;
    if (p->dgain) {
        rc = op_launch(ctx, "k_norm_dgain", k_norm_dgain, dim3((unsigned)((P.cols + 31) / 32)), DGAIN_WARPS * 32, stream, (const float *)P.part, P.ld_part, plan.slots,
                       p->dgain, P.cols, p->accumulate ? 1 : 0);
        if (rc) return rc;
    }
    return op_workspace_done(ctx, use);
}

// ------------------------------------------------------------------ encoders
typedef void (*Encoder)(EncodeParams);
template <class T, int NG> Encoder row_encoder_as(int access) { return access == 8 ? k_encode_rows<T, 8, NG> : access == 4 ? k_encode_rows<T, 4, NG> : k_encode_rows<T, 1, NG>; }
template <class T> Encoder row_encoder_of(int access, int ng) { return ng == 4 ? row_encoder_as<T, 4>(access) : ng == 2 ? row_encoder_as<T, 2>(access) : row_encoder_as<T, 1>(access); }
template <class T> Encoder block_encoder_of(int access) { return access == 8 ? k_encode_blocks<T, 8> : access == 4 ? k_encode_blocks<T, 4> : k_encode_blocks<T, 1>; }
Encoder row_encoder(int dtype, int access, int ng)
{
    return dtype == CONDENSA_DTYPE_BF16 ? row_encoder_of<__nv_bfloat16>(access, ng) : dtype == CONDENSA_DTYPE_FP16 ? row_encoder_of<__half>(access, ng) : row_encoder_of<float>(access, ng);
}
Encoder block_encoder(int dtype, int access)
{
    return dtype == CONDENSA_DTYPE_BF16 ? block_encoder_of<__nv_bfloat16>(access) : dtype == CONDENSA_DTYPE_FP16 ? block_encoder_of<__half>(access) : block_encoder_of<float>(access);
}
int encode_rows(condensa_ctx *ctx, const void *x, long long ldx, long long rows, long long cols, int dtype, const condensa_coded *out, cudaStream_t stream)
{
    if (!out) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "out is NULL");
    if (!op_known_type(dtype)) return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "dtype must be CONDENSA_DTYPE_FP32, _FP16 or _BF16");
    OpArgs a(ctx);
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
    P.groups = (u32)((P.cols + GROUP - 1) / GROUP);
    RowRuns plan;
    if (!plan_row_runs(rows, P.groups, THREADS / GROUP_LANES, plan)) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "too many groups for one launch");
    P.runs = plan.runs;
    P.reciprocal = plan.reciprocal;
    CU_TRY(ctx, cudaSetDevice(ctx->device));
    return op_launch(ctx, "k_encode_rows", row_encoder(dtype, op_access(x, ldx, e, cols), plan.groups_of_run), dim3((unsigned)plan.grid), THREADS, stream, P);
}

int encode_blocks(condensa_ctx *ctx, const void *w, long long ldw, long long n, long long k, int dtype, const condensa_coded *out, float *theta, long long ld_theta,
                  cudaStream_t stream)
{
    if (!out) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "out is NULL");
    if (!op_known_type(dtype)) return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "dtype must be CONDENSA_DTYPE_FP32, _FP16 or _BF16");
    if (n < 1 || k < 1) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "n and k must be positive");
    if (n > OP_MAX_WIDTH || k > OP_MAX_WIDTH) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "n and k must not exceed 2^22");
    OpArgs a(ctx);
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
    P.groups = (u32)((P.cols + GROUP - 1) / GROUP);
    CU_TRY(ctx, cudaSetDevice(ctx->device));
    return op_launch(ctx, "k_encode_blocks", block_encoder(dtype, std::min(op_access(w, ldw, e, k), op_access(theta, ld_theta, 4, k))),
                     dim3((unsigned)((n + GROUP - 1) / GROUP * P.groups)), ENC_BLOCK, stream, P);
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
