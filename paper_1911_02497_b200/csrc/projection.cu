// Host side of the products with a projection in 8 bits: argument checks, tensor maps, launches.
#include <new>

#include "op_args.h"
#include "projection.cuh"

using namespace cs;

static_assert(CONDENSA_CODE_GROUP == GROUP, "columns that share a scale");

namespace {

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// (an entry point of the driver: the same for the process)
EncodeTiled find_encode_tiled()
{
    void *p = nullptr;
    cudaDriverEntryPointQueryResult got = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &got) != cudaSuccess) {
        cudaGetLastError();
        return nullptr;
    }
    return got == cudaDriverEntryPointSuccess ? (EncodeTiled)p : nullptr;
}

// Boxes of 128 columns x `high` rows of a code matrix, zero outside, swizzled in shared memory by 128 bytes.
int code_map(condensa_ctx *ctx, CUtensorMap &map, const condensa_coded &c, long long rows, long long cols, int high)
{
    static const EncodeTiled f = find_encode_tiled();
    if (!f) return fail(ctx, CONDENSA_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
    const cuuint64_t dim[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)c.ld};
    const cuuint32_t box[2] = {GROUP, (cuuint32_t)high}, step[2] = {1, 1};
    const CUresult e = f(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, c.codes, dim, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (e != CUDA_SUCCESS) return fail(ctx, CONDENSA_ERR_CUDA, "cuTensorMapEncodeTiled: error %d", (int)e);
    return CONDENSA_OK;
}

typedef void (*Kernel)(ProjectionParams);

constexpr int PJ_SMEM_MOST = 227 * 1024, PJ_SMEM_HALF = 113 * 1024;

struct Variant {
    Kernel f;
    int wide, threads, fixed, stages;       // output columns of a tile; shared memory beside the ring; most stages
    bool sums;                              // the ring holds a tile's sums in the end
};

template <class T, bool TRANS>
Variant variant_of(const ProjectionCut &s)
{
    if (!s.pair) return {k_projection<T, TRANS>, PJ_WIDE, 128, PJ_PAD + PJ_SLOTS * PJ_SCALES, PJ_STAGES, true};
    const int fixed = PJ_PAD + PJ_SLOTS * PP_SCALES + PP_OUT;
    if (s.parts > 1) return {k_projection_pair<T, TRANS, true>, 2 * PJ_WIDE, PP_THREADS, fixed, PP_STAGES, true};
    return {k_projection_pair<T, TRANS, false>, 2 * PJ_WIDE, PP_THREADS, fixed, PP_STAGES, false};
}

Variant variant_of(int dtype, bool trans, const ProjectionCut &s)
{
    return dtype == CONDENSA_DTYPE_BF16 ? (trans ? variant_of<__nv_bfloat16, true>(s) : variant_of<__nv_bfloat16, false>(s))
                                        : (trans ? variant_of<__half, true>(s) : variant_of<__half, false>(s));
}

int allow_smem(condensa_ctx *ctx, Kernel k)
{
    for (const void *f : ctx->op_smem_set)
        if (f == (const void *)k) return CONDENSA_OK;
    CU_TRY(ctx, cudaFuncSetAttribute((const void *)k, cudaFuncAttributeMaxDynamicSharedMemorySize, PJ_SMEM_MOST - 1024));
    ctx->op_smem_set.push_back((const void *)k);
    return CONDENSA_OK;
}

// Clusters of `n` CTAs, one on an SM, that the device holds at once.
int resident_clusters(condensa_ctx *ctx, const Variant &v, int n, int &count)
{
    for (const condensa_ctx::ClusterFit &f : ctx->cluster_fit)
        if (f.f == (const void *)v.f && f.size == n) {
            count = f.count;
            return CONDENSA_OK;
        }
    const int rc = allow_smem(ctx, v.f);
    if (rc) return rc;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)n);
    cfg.blockDim = dim3((unsigned)v.threads);
    cfg.dynamicSmemBytes = (size_t)(PJ_SMEM_MOST - 1024);
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)n;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    count = 0;
    CU_TRY(ctx, cudaOccupancyMaxActiveClusters(&count, (const void *)v.f, &cfg));
    ctx->cluster_fit.push_back({(const void *)v.f, n, count});
    return CONDENSA_OK;
}

int run(condensa_ctx *ctx, const condensa_projection *w, const condensa_coded *x, long long rows, void *y, long long ldy, int dtype, bool trans,
        cudaStream_t stream)
{
    if (!w || !x) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "an operand is NULL");
    if (dtype != CONDENSA_DTYPE_FP16 && dtype != CONDENSA_DTYPE_BF16) return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "dtype must be CONDENSA_DTYPE_FP16 or _BF16");
    if (w->n < 1 || w->k < 1) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "n and k must be positive");
    if (w->n > OP_MAX_WIDTH || w->k > OP_MAX_WIDTH) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "n and k must not exceed 2^22");
    const long long depth = trans ? w->n : w->k, width = trans ? w->k : w->n;
    OpArgs a(ctx);
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
    P.access = op_access(y, ldy, 2, width);
    const int quads = (P.groups + PJ_QUAD - 1) / PJ_QUAD;
    ProjectionCut shape;
    rc = choose_cut(rows, width, P.groups, ctx->num_sms, [&](const ProjectionCut &s, int n, int &count) {
        return resident_clusters(ctx, variant_of(dtype, trans, s), n, count);
    }, shape);
    if (rc) return rc;
    const Variant v = variant_of(dtype, trans, shape);
    const int high = shape.pair ? shape.tile / 2 : shape.tile, stage = PJ_A + high * GROUP, deepest = (quads + shape.parts - 1) / shape.parts * PJ_QUAD;
    P.tile = shape.tile;
    P.blocks = (int)((width + v.wide - 1) / v.wide);
    const long long tiles = (rows + P.tile - 1) / P.tile * P.blocks, ctas = std::min(tiles * shape.parts, shape.clusters) * (shape.pair ? 2 : 1);
    if (tiles * shape.parts > 0x3FFFFFFFll) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "too many tiles for one launch");
    P.tiles = (int)tiles;
    // as many stages as there is room for (a CTA by itself shares its SM where there are more of them than SMs)
    const int fixed = v.fixed + 1024, room = (!shape.pair && ctas > ctx->num_sms ? PJ_SMEM_HALF : PJ_SMEM_MOST) - fixed;
    P.stages = std::min(std::min(v.stages, deepest), room / stage);
    P.ring = std::max(P.stages * stage, v.sums ? P.tile * PJ_WIDE * 4 : 0);
    P.columns = 32;
    while (P.columns < (u32)P.tile + PJ_SLOTS * 8) P.columns *= 2;
    if ((rc = code_map(ctx, P.w, w->code, w->n, w->k, PJ_WIDE)) != 0) return rc;
    if ((rc = code_map(ctx, P.x, *x, rows, depth, high)) != 0) return rc;
    if ((rc = allow_smem(ctx, v.f)) != 0) return rc;
    // A CTA of a pair has the SM to itself: it waits for its partner while it holds tensor memory, and two pairs that held it on one
    // SM each would wait for one another. (A CTA by itself gives it back ahead of any such wait.)
    PdlLaunch l(ctx, 1, v.threads, shape.pair ? (size_t)(PJ_SMEM_MOST - 1024) : (size_t)(v.fixed + P.ring), stream);
    l.cfg.gridDim = dim3((unsigned)ctas);
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)(shape.parts * (shape.pair ? 2 : 1));
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1] = l.attr;
    l.cfg.attrs = at;
    l.cfg.numAttrs += 1;
    const int pa_ = prof_begin(ctx, trans ? "k_projection_back" : "k_projection", stream);
    CU_TRY(ctx, cudaLaunchKernelEx(&l.cfg, v.f, P));
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
