// What each type's source file compiles of the norm: the choice of a kernel, and its launch.
#pragma once
#include "norm_launch.cuh"

using namespace cs;

namespace {

// CTAs of a kernel that an SM holds; allows it its shared memory.
int resident_ctas(condensa_ctx *ctx, const void *f, int block, int smem, int &count)
{
    for (const condensa_ctx::ClusterFit &k : ctx->cluster_fit)
        if (k.f == f && k.size == 0) {
            count = k.count;
            return CONDENSA_OK;
        }
    if (smem) CU_TRY(ctx, cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    count = 0;
    CU_TRY(ctx, cudaOccupancyMaxActiveBlocksPerMultiprocessor(&count, f, block, (size_t)smem));
    if (count < 1) return fail(ctx, CONDENSA_ERR_INTERNAL, "a kernel of the norm does not fit an SM");
    ctx->cluster_fit.push_back({f, 0, count});
    return CONDENSA_OK;
}

constexpr int LONG_TPR = 512;           // threads of a row that is read twice

template <class T, int A, int TPR, int NV>
int forward_as(condensa_ctx *ctx, const NormParams &P, cudaStream_t stream)
{
    constexpr int ROWS = RowThreads<TPR>::ROWS;
    return op_launch(ctx, "k_norm_forward", k_norm_forward<T, A, TPR, NV>, dim3((unsigned)((P.rows + ROWS - 1) / ROWS)), RowThreads<TPR>::BLOCK, stream, P);
}

// The threads of a row: as many as hold it with one or two eights each. With steps of powers of two alone, where up to half of the threads
// have nothing to do: 8000 x 1500 bf16 21 us instead of 19, 4000 x 6000 42 instead of 36; backward 4000 x 6000 56 instead of 43, 2000 x 9999
// 127 instead of 85.
template <class T, int A>
int forward_of(condensa_ctx *ctx, const NormParams &P, cudaStream_t stream)
{
    const int eights = (P.cols + 7) / 8;
    if (eights > 2048)
        return op_launch(ctx, "k_norm_forward_long", k_norm_forward_long<T, A, LONG_TPR>, dim3((unsigned)P.rows), LONG_TPR, stream, P);
    return eights <= 32   ? forward_as<T, A, 32, 1>(ctx, P, stream)
         : eights <= 64   ? forward_as<T, A, 32, 2>(ctx, P, stream)
         : eights <= 128  ? forward_as<T, A, 128, 1>(ctx, P, stream)
         : eights <= 192  ? forward_as<T, A, 96, 2>(ctx, P, stream)
         : eights <= 256  ? forward_as<T, A, 128, 2>(ctx, P, stream)
         : eights <= 384  ? forward_as<T, A, 192, 2>(ctx, P, stream)
         : eights <= 512  ? forward_as<T, A, 256, 2>(ctx, P, stream)
         : eights <= 768  ? forward_as<T, A, 384, 2>(ctx, P, stream)
         : eights <= 1024 ? forward_as<T, A, 512, 2>(ctx, P, stream)
         : eights <= 1536 ? forward_as<T, A, 768, 2>(ctx, P, stream)
                          : forward_as<T, A, 1024, 2>(ctx, P, stream);
}

template <class T, int A, int TPR, int NV>
int backward_as(condensa_ctx *ctx, const NormBackParams &P, NormBackPlan &plan, bool run, cudaStream_t stream)
{
    constexpr int ROWS = RowThreads<TPR>::ROWS, BLOCK = RowThreads<TPR>::BLOCK;
    auto k = k_norm_backward<T, A, TPR, NV>;
    constexpr int SMEM = BackRing<T, A, TPR, NV>::SMEM;
    if (run) return op_launch_smem(ctx, "k_norm_backward", k, dim3((unsigned)plan.grid), BLOCK, SMEM, stream, P);
    int fit = 1;
    const int rc = resident_ctas(ctx, (const void *)k, BLOCK, SMEM, fit);
    if (rc) return rc;
    plan.grid = stream_grid(ctx, (P.rows + ROWS - 1) / ROWS, fit);
    plan.slots = plan.grid * ROWS;
    return CONDENSA_OK;
}

template <class T, int A>
int backward_of(condensa_ctx *ctx, const NormBackParams &P, NormBackPlan &plan, bool run, cudaStream_t stream)
{
    const int eights = (P.cols + 7) / 8;
    // (fp32 operands of longer rows leave no room for two stages)
    if (eights > (sizeof(T) == 4 ? 1024 : 2048)) {
        const unsigned strips = (unsigned)((eights + THREADS - 1) / THREADS);
        if (!run) {
            plan.grid = (int)std::min(P.rows, std::max(1ll, 4ll * ctx->num_sms / strips));
            plan.slots = plan.grid;
            return CONDENSA_OK;
        }
        int rc = CONDENSA_OK;
        if (P.part) rc = op_launch(ctx, "k_norm_dgain_long", k_norm_dgain_long<T, A>, dim3(strips, (unsigned)plan.grid), THREADS, stream, P);
        if (rc || (!P.dx && !P.codes)) return rc;
        return op_launch(ctx, "k_norm_backward_long", k_norm_backward_long<T, A, LONG_TPR>, dim3((unsigned)P.rows), LONG_TPR, stream, P);
    }
    if constexpr (sizeof(T) == 2) {
        if (eights > 1536) return backward_as<T, A, 1024, 2>(ctx, P, plan, run, stream);
        if (eights > 1024) return backward_as<T, A, 768, 2>(ctx, P, plan, run, stream);
    }
    return eights <= 32  ? backward_as<T, A, 32, 1>(ctx, P, plan, run, stream)
         : eights <= 64  ? backward_as<T, A, 32, 2>(ctx, P, plan, run, stream)
         : eights <= 128 ? backward_as<T, A, 128, 1>(ctx, P, plan, run, stream)
         : eights <= 256 ? backward_as<T, A, 128, 2>(ctx, P, plan, run, stream)      // (96 threads: 32 instead of 28 us for 8192 x 1500 in bf16)
         : eights <= 384 ? backward_as<T, A, 192, 2>(ctx, P, plan, run, stream)
         : eights <= 512 ? backward_as<T, A, 256, 2>(ctx, P, plan, run, stream)
         : eights <= 768 ? backward_as<T, A, 384, 2>(ctx, P, plan, run, stream)
                         : backward_as<T, A, 512, 2>(ctx, P, plan, run, stream);
}

}  // namespace

template <class T>
int norm_forward_launch(condensa_ctx *ctx, const NormParams &P, int access, cudaStream_t stream)
{
    return access == 8 ? forward_of<T, 8>(ctx, P, stream) : access == 4 ? forward_of<T, 4>(ctx, P, stream) : forward_of<T, 1>(ctx, P, stream);
}

template <class T>
int norm_backward_launch(condensa_ctx *ctx, const NormBackParams &P, NormBackPlan &plan, int access, bool run, cudaStream_t stream)
{
    return access == 8 ? backward_of<T, 8>(ctx, P, plan, run, stream)
         : access == 4 ? backward_of<T, 4>(ctx, P, plan, run, stream) : backward_of<T, 1>(ctx, P, plan, run, stream);
}
