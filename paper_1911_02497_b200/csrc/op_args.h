// Argument checks that the 8-bit operators and the norm share. Host code.
#pragma once
#include "ctx.cuh"

inline bool op_known_type(int t) { return t == CONDENSA_DTYPE_FP32 || t == CONDENSA_DTYPE_FP16 || t == CONDENSA_DTYPE_BF16; }
inline int op_type_bytes(int t) { return t == CONDENSA_DTYPE_FP32 ? 4 : 2; }

constexpr long long OP_MAX_WIDTH = 1ll << 22, OP_MAX_ROWS = (1ll << 31) - 256;

// The matrices of a call: each is checked as it is noted, and at last whether an output meets anything else.
struct OpArgs {
    condensa_ctx *ctx;
    std::vector<Interval> iv;
    std::vector<RowRange> rows;

    explicit OpArgs(condensa_ctx *c) : ctx(c)
    {
        iv.reserve(4);
        rows.reserve(8);
    }
    int matrix(const char *name, const void *p, long long ld, long long n, long long width, int e, bool out)
    {
        if (!p) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "%s is NULL", name);
        if ((uintptr_t)p % e) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "%s is not aligned to its type", name);
        if (ld < width) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "%s: rows of %lld values lie %lld apart", name, width, ld);
        if (ld > (1ll << 39) || n - 1 > (1ll << 56) / ld) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "%s: %lld rows %lld apart leave the address space", name, n, ld);
        rows.push_back({(uintptr_t)p, (uintptr_t)(width * e), (uintptr_t)(ld * e), (uintptr_t)n, out});
        return CONDENSA_OK;
    }
    void array(const void *p, long long bytes, bool out)
    {
        if (p && bytes > 0) iv.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, out});
    }
    // An 8-bit matrix of n rows with a scale for every `high` of them.
    int coded(const char *name, const condensa_coded &c, long long n, long long cols, int high, bool out)
    {
        const long long groups = (cols + CONDENSA_CODE_GROUP - 1) / CONDENSA_CODE_GROUP;
        if (!c.codes || !c.scales) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "%s: codes or scales are NULL", name);
        if ((uintptr_t)c.codes % 16 || c.ld % 16) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "%s: codes must be 16-byte aligned, their rows a multiple of 16 bytes apart", name);
        if ((uintptr_t)c.scales % 4 || c.ld_scales % 4) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "%s: scales must be 4-byte aligned, their rows a multiple of 4 bytes apart", name);
        int rc = matrix(name, c.codes, c.ld, n, cols, 1, out);
        if (rc) return rc;
        return matrix(name, c.scales, c.ld_scales, (n + high - 1) / high, groups, 1, out);
    }
    int sizes(long long n, long long cols)
    {
        if (n < 0 || cols < 1) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "rows must not be negative, and columns positive");
        if (n > OP_MAX_ROWS || cols > OP_MAX_WIDTH) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "at most 2^31 - 256 rows and 2^22 columns");
        return CONDENSA_OK;
    }
    int apart()
    {
        return rows_clash(iv, rows) ? fail(ctx, CONDENSA_ERR_INVALID_ARG, "an output buffer overlaps another buffer of the call") : CONDENSA_OK;
    }
};

// Values of `e` bytes that an access to rows `ld` apart may take at once: 8, 4 or 1 (rows of `cols`).
inline int op_access(const void *p, long long ld, int e, long long cols)
{
    if (!p) return 8;
    const uintptr_t bits = (uintptr_t)p | (uintptr_t)(ld * e);
    return bits % 16 == 0 && cols % 8 == 0 ? 8 : bits % (4 * e) == 0 && cols % 4 == 0 ? 4 : 1;
}

// A launch that may start while the kernel ahead of it ends: every kernel launched so waits for that one before it reads or
// writes anything.
template <class... A>
inline int op_launch_smem(condensa_ctx *ctx, const char *name, void (*k)(A...), dim3 grid, int block, size_t smem, cudaStream_t stream, A... args)
{
    PdlLaunch l(ctx, 1, block, smem, stream);
    l.cfg.gridDim = grid;
    const int pa_ = prof_begin(ctx, name, stream);
    CU_TRY(ctx, cudaLaunchKernelEx(&l.cfg, k, args...));
    ctx->launches += 1;
    prof_end(ctx, pa_, stream);
    return CONDENSA_OK;
}
template <class... A>
inline int op_launch(condensa_ctx *ctx, const char *name, void (*k)(A...), dim3 grid, int block, cudaStream_t stream, A... args)
{
    return op_launch_smem(ctx, name, k, grid, block, 0, stream, args...);
}
