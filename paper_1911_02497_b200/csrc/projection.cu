// Host side of the products with a projection in 8 bits: argument checks, tensor maps, launches.
#include <new>

#include "op_args.h"
#include "projection.cuh"

using namespace cs;

static_assert(CONDENSA_CODE_GROUP == GROUP, "columns that share a scale");

namespace {

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int encode_tiled(condensa_ctx *ctx, EncodeTiled &f)
{
    static EncodeTiled known = nullptr;         // (an entry point of the driver: the same for the process)
    if (!known) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult got = cudaDriverEntryPointSymbolNotFound;
        CU_TRY(ctx, cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &got));
        if (got != cudaDriverEntryPointSuccess || !p) return fail(ctx, CONDENSA_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
        known = (EncodeTiled)p;
    }
    f = known;
    return CONDENSA_OK;
}

// Boxes of 128 columns x `high` rows of a code matrix, zero outside, swizzled in shared memory by 128 bytes.
int code_map(condensa_ctx *ctx, CUtensorMap &map, const condensa_coded &c, long long rows, long long cols, int high)
{
    EncodeTiled f;
    const int rc = encode_tiled(ctx, f);
    if (rc) return rc;
    const cuuint64_t dim[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)c.ld};
    const cuuint32_t box[2] = {GROUP, (cuuint32_t)high}, step[2] = {1, 1};
    const CUresult e = f(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, c.codes, dim, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (e != CUDA_SUCCESS) return fail(ctx, CONDENSA_ERR_CUDA, "cuTensorMapEncodeTiled: error %d", (int)e);
    return CONDENSA_OK;
}

typedef void (*Kernel)(ProjectionParams);

constexpr int PJ_SMEM_MOST = 227 * 1024, PJ_SMEM_HALF = 113 * 1024, PJ_MAX_PARTS = 8;

int run(condensa_ctx *ctx, const condensa_projection *w, const condensa_coded *x, long long rows, void *y, long long ldy, int dtype, bool trans,
        cudaStream_t stream)
{
    if (!w || !x) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "an operand is NULL");
    if (dtype != CONDENSA_DTYPE_FP16 && dtype != CONDENSA_DTYPE_BF16) return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "dtype must be CONDENSA_DTYPE_FP16 or _BF16");
    if (w->n < 1 || w->k < 1) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "n and k must be positive");
    if (w->n > OP_MAX_WIDTH || w->k > OP_MAX_WIDTH) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "n and k must not exceed 2^22");
    const long long depth = trans ? w->n : w->k, width = trans ? w->k : w->n;
    OpArgs a{ctx};
    int rc = a.sizes(rows, depth);
    if (rc || rows == 0) return rc;
    if ((rc = a.coded("w", w->code, w->n, w->k, GROUP, false)) != 0) return rc;
    if ((rc = a.coded(trans ? "dy" : "x", *x, rows, depth, 1, false)) != 0) return rc;
    if ((rc = a.matrix(trans ? "dx" : "y", y, ldy, rows, width, 2, true)) != 0) return rc;
    if ((rc = a.apart()) != 0) return rc;
    CU_TRY(ctx, cudaSetDevice(ctx->device));
    ProjectionParams P;
    memset(&P, 0, sizeof(P));
    P.w_scales = w->code.scales;
    P.w_depth = trans ? w->code.ld_scales : 1;
    P.w_wide = trans ? 1 : w->code.ld_scales;
    P.x_scales = x->scales;
    P.ld_xs = x->ld_scales;
    P.out = y;
    P.ldo = ldy;
    P.rows = rows;
    P.width = (int)width;
    P.groups = (int)((depth + GROUP - 1) / GROUP);
    P.blocks = (int)((width + PJ_WIDE - 1) / PJ_WIDE);
    P.access = op_access(y, ldy, 2, width);
    // equal tiles of rows
    const long long tiles = (rows + PJ_MAX_TILE - 1) / PJ_MAX_TILE;
    P.tile = (int)(((rows + tiles - 1) / tiles + 15) / 16 * 16);
    const int quads = (P.groups + PJ_QUAD - 1) / PJ_QUAD;
    long long ctas = tiles * P.blocks;
    int parts = 1;
    while (parts < PJ_MAX_PARTS && parts < quads && ctas * (parts + 1) <= ctx->num_sms) ++parts;
    ctas *= parts;
    if (ctas > 0x7FFFFFFFll) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "too many tiles for one launch");
    const int stage = PJ_A + P.tile * GROUP, fixed = PJ_PAD + PJ_SLOTS * PJ_SCALES + 1024;
    const int room = (ctas > ctx->num_sms ? PJ_SMEM_HALF : PJ_SMEM_MOST) - fixed;
    const int deepest = (quads + parts - 1) / parts * PJ_QUAD;
    P.stages = std::min(std::min(PJ_STAGES, deepest), room / stage);
    P.ring = std::max(P.stages * stage, P.tile * PJ_WIDE * 4);
    P.columns = 32;
    while (P.columns < (u32)P.tile + 16) P.columns *= 2;
    if ((rc = code_map(ctx, P.w, w->code, w->n, w->k, PJ_WIDE)) != 0) return rc;
    if ((rc = code_map(ctx, P.x, *x, rows, depth, P.tile)) != 0) return rc;
    const Kernel k = dtype == CONDENSA_DTYPE_BF16 ? (trans ? k_projection<__nv_bfloat16, true> : k_projection<__nv_bfloat16, false>)
                                                  : (trans ? k_projection<__half, true> : k_projection<__half, false>);
    bool known = false;
    for (const void *f : ctx->op_smem_set) known = known || f == (const void *)k;
    if (!known) {
        CU_TRY(ctx, cudaFuncSetAttribute((const void *)k, cudaFuncAttributeMaxDynamicSharedMemorySize, PJ_SMEM_MOST - 1024));
        ctx->op_smem_set.push_back((const void *)k);
    }
    PdlLaunch l(ctx, 1, 128, (size_t)(PJ_PAD + P.ring + PJ_SLOTS * PJ_SCALES), stream);
    l.cfg.gridDim = dim3((unsigned)ctas);
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)parts;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1] = l.attr;
    l.cfg.attrs = at;
    l.cfg.numAttrs += 1;
    const int pa_ = prof_begin(ctx, trans ? "k_projection_back" : "k_projection", stream);
    CU_TRY(ctx, cudaLaunchKernelEx(&l.cfg, k, P));
    ctx->launches += 1;
    prof_end(ctx, pa_, stream);
    return CONDENSA_OK;
}

}  // namespace

extern "C" {

int condensa_projection_forward(condensa_ctx *ctx, const condensa_projection *w, const condensa_coded *x, int64_t rows, void *y, int64_t ldy, int dtype,
                                void *stream)
{
    if (!ctx) return CONDENSA_ERR_INVALID_ARG;
    try {
        return run(ctx, w, x, rows, y, ldy, dtype, false, (cudaStream_t)stream);
    } catch (const std::bad_alloc &) {
        return fail(ctx, CONDENSA_ERR_WORKSPACE, "out of host memory");
    }
}

int condensa_projection_backward(condensa_ctx *ctx, const condensa_projection *w, const condensa_coded *dy, int64_t rows, void *dx, int64_t lddx, int dtype,
                                 void *stream)
{
    if (!ctx) return CONDENSA_ERR_INVALID_ARG;
    try {
        return run(ctx, w, dy, rows, dx, lddx, dtype, true, (cudaStream_t)stream);
    } catch (const std::bad_alloc &) {
        return fail(ctx, CONDENSA_ERR_WORKSPACE, "out of host memory");
    }
}

}  // extern "C"
