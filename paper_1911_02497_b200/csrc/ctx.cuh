// What every source file of the host side shares: the context, error texts, per-kernel timing,
// launch helpers, the workspace of the operators.
#pragma once
#include "../../include/condensa_cstep.h"

#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <string>
#include <vector>

#include "common.cuh"
#include "op_workspace.h"
#include "ranges.h"

using cs::Ctl;

inline std::string g_create_error;   // text of a failure without a context

struct KernelInfo {
    int occ = 0;     // CTAs per SM
};

struct DeviceMirror {   // device copies used by condensa_cstep_host
    char *buf = nullptr;
    size_t bytes = 0;
};

struct condensa_ctx {
    int device = 0;
    int num_sms = 0;
    bool coop = false;
    std::string err;
    char *ws = nullptr;
    size_t ws_bytes = 0;
    char *h_stage = nullptr;        // pinned staging of the descriptor upload
    size_t h_stage_bytes = 0;
    cudaEvent_t stage_ev = nullptr;
    cudaEvent_t tail_ev = nullptr;  // recorded behind the last kernel of every call
    bool tail_recorded = false;
    uint64_t seed = 0;              // sample positions of the single-pass path
    std::vector<char> last_upload;  // what the device descriptor area holds now
    char *last_upload_dst = nullptr;
    int64_t launches = 0;
    cudaStream_t last_stream = nullptr;
    bool has_result = false;
    Ctl *ctl = nullptr;
    int occ_select[4] = {0, 0, 0, 0};
    int occ_stream = 0;
    int occ_filter = 0;
    int occ_prune_small = 0;        // resident CTAs per SM of the register-resident small-list kernel
    bool small_smem_set = false;    // dynamic shared memory limit of k_select_small raised on this device
    bool block_smem_set = false;    // the same for the tiled block kernel
    size_t blockg_smem_set = 0;     // ... and for the tiled bh x bw kernel (bytes it has been allowed so far)
    DeviceMirror mirror;
    // optional per-kernel timing (event pair around every launch)
    bool prof_on = false;
    std::vector<cudaEvent_t> prof_ev;       // start/stop pairs
    std::vector<int> prof_name;             // index into prof_names per pair
    std::vector<std::string> prof_names;
    size_t prof_used = 0;                   // pairs recorded since the last read
    std::vector<double> prof_ms;            // accumulated per name
    std::vector<int64_t> prof_cnt;
    struct ClusterFit { const void *f; int size, count; };
    std::vector<ClusterFit> cluster_fit;    // clusters of a kernel that the device holds at once; size 0: CTAs of it that an SM holds
    std::vector<const void *> op_smem_set;  // kernels of the adapters and of the 8-bit products whose shared memory limit has been raised on this device
    OpWorkspace op;                         // of the list operators, the adapters and the norm's gradient; apart from the C-step's
};

inline int fail(condensa_ctx *c, int code, const char *fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    if (c) c->err = buf; else g_create_error = buf;
    return code;
}

#define CU_TRY(ctx, call)                                                                   \
    do {                                                                                    \
        cudaError_t e_ = (call);                                                            \
        if (e_ != cudaSuccess)                                                              \
            return fail(ctx, CONDENSA_ERR_CUDA, "%s: %s", #call, cudaGetErrorString(e_));   \
    } while (0)

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline int stream_grid(condensa_ctx *ctx, long long n_items, int occ)
{
    long long g = (long long)ctx->num_sms * occ;
    if (g > n_items) g = n_items;
    if (g < 1) g = 1;
    return (int)g;
}

inline int prof_begin(condensa_ctx *ctx, const char *name, cudaStream_t stream)
{
    if (!ctx->prof_on) return 0;
    if (ctx->prof_used * 2 + 2 > ctx->prof_ev.size()) {
        for (int i = 0; i < 2; ++i) {
            cudaEvent_t e;
            if (cudaEventCreate(&e) != cudaSuccess) return 0;
            ctx->prof_ev.push_back(e);
        }
    }
    int id = -1;
    for (size_t i = 0; i < ctx->prof_names.size(); ++i)
        if (ctx->prof_names[i] == name) id = (int)i;
    if (id < 0) {
        id = (int)ctx->prof_names.size();
        ctx->prof_names.push_back(name);
        ctx->prof_ms.push_back(0.0);
        ctx->prof_cnt.push_back(0);
    }
    if (ctx->prof_name.size() <= ctx->prof_used) ctx->prof_name.resize(ctx->prof_used + 1);
    ctx->prof_name[ctx->prof_used] = id;
    cudaEventRecord(ctx->prof_ev[ctx->prof_used * 2], stream);
    return 1;
}

inline void prof_end(condensa_ctx *ctx, int active, cudaStream_t stream)
{
    if (!active) return;
    cudaEventRecord(ctx->prof_ev[ctx->prof_used * 2 + 1], stream);
    ctx->prof_used += 1;
}

// Folds the recorded event pairs into the per-kernel totals (synchronises).
inline void prof_collect(condensa_ctx *ctx)
{
    for (size_t i = 0; i < ctx->prof_used; ++i) {
        float ms = 0.0f;
        cudaEventSynchronize(ctx->prof_ev[2 * i + 1]);
        if (cudaEventElapsedTime(&ms, ctx->prof_ev[2 * i], ctx->prof_ev[2 * i + 1]) == cudaSuccess) {
            ctx->prof_ms[ctx->prof_name[i]] += ms;
            ctx->prof_cnt[ctx->prof_name[i]] += 1;
        }
    }
    ctx->prof_used = 0;
}

// Launch configuration with the programmatic-dependent-launch attribute (dropped while every
// kernel is bracketed by an event pair: nothing can overlap then).
struct PdlLaunch {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr;
    PdlLaunch(const condensa_ctx *ctx, int grid, int block, size_t smem, cudaStream_t stream)
    {
        memset(&cfg, 0, sizeof(cfg));
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cfg.gridDim = dim3((unsigned)grid);
        cfg.blockDim = dim3((unsigned)block);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = stream;
        cfg.attrs = &attr;
        cfg.numAttrs = ctx->prof_on ? 0 : 1;
    }
};

#define LAUNCH_CHECK(ctx)                                                                    \
    do {                                                                                     \
        cudaError_t e_ = cudaGetLastError();                                                 \
        if (e_ != cudaSuccess)                                                               \
            return fail(ctx, CONDENSA_ERR_CUDA, "kernel launch: %s", cudaGetErrorString(e_)); \
        ctx->launches += 1;                                                                  \
    } while (0)

// Room for `bytes` in the operators' workspace (op_workspace.h); `use` lives to the end of the call.
inline int op_workspace(condensa_ctx *ctx, size_t bytes, cudaStream_t stream, OpWorkspaceUse &use)
{
    cudaError_t e = cudaSuccess;
    switch (op_workspace_take(ctx->op, bytes, stream, e, use)) {
    case OP_WS_OK: return CONDENSA_OK;
    case OP_WS_CAPTURE:
        return fail(ctx, CONDENSA_ERR_WORKSPACE, "the workspace must grow, which a stream capture does not allow: make the call once before");
    case OP_WS_MEMORY: return fail(ctx, CONDENSA_ERR_WORKSPACE, "cannot allocate a workspace for %zu bytes: %s", bytes, cudaGetErrorString(e));
    default: return fail(ctx, CONDENSA_ERR_CUDA, "workspace: %s", cudaGetErrorString(e));
    }
}

// Behind the last launch of a call that may have used it.
inline int op_workspace_done(condensa_ctx *ctx, OpWorkspaceUse &use)
{
    CU_TRY(ctx, op_workspace_leave(use));
    return CONDENSA_OK;
}
