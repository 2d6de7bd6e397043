// Workspace of the list operators and the adapters (partial sums, coefficients, matrices laid out anew). Host code
// over the CUDA runtime alone.
#pragma once
#include <cuda_runtime_api.h>

#include <cstddef>
#include <vector>

struct OpWorkspace {
    char *p = nullptr;
    size_t bytes = 0;
    cudaEvent_t ev = nullptr;               // recorded behind the last call that used it
    cudaStream_t stream = nullptr;          // of that call
    bool recorded = false;
    bool capturing = false;                 // the call under way is being captured
    bool in_graph = false;                  // a captured call was given this block
    std::vector<char *> kept;               // outgrown blocks whose addresses graphs hold
};

enum OpWorkspaceStatus { OP_WS_OK, OP_WS_CUDA, OP_WS_CAPTURE, OP_WS_MEMORY };

// Room for `want` bytes, ordered behind its last user on another stream. The first 256 bytes hold counters that are
// zero between calls. Growing waits for the device once, so it cannot happen inside a stream capture; a captured call
// is not ordered behind other streams (the event would belong to work outside the graph): its replays must not overlap
// other calls. A graph holds the block's address for as long as it may be replayed, so a block that a capture
// was given is not freed when it is outgrown, but with the context. `e`: the CUDA error behind a status that is not OP_WS_OK.
inline OpWorkspaceStatus op_workspace_take(OpWorkspace &w, size_t want, cudaStream_t stream, cudaError_t &e)
{
    cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
    if ((e = cudaStreamIsCapturing(stream, &st)) != cudaSuccess) return OP_WS_CUDA;
    w.capturing = st != cudaStreamCaptureStatusNone;
    if (w.capturing) {
        if (want > w.bytes) return OP_WS_CAPTURE;
        w.in_graph = true;
        return OP_WS_OK;
    }
    if (!w.ev && (e = cudaEventCreateWithFlags(&w.ev, cudaEventDisableTiming)) != cudaSuccess) return OP_WS_CUDA;
    if (want > w.bytes) {
        if ((e = cudaDeviceSynchronize()) != cudaSuccess) return OP_WS_CUDA;
        if (w.in_graph) w.kept.push_back(w.p);
        else if (w.p) cudaFree(w.p);
        w.p = nullptr;
        w.bytes = 0;
        w.in_graph = false;
        w.recorded = false;
        const size_t mib = 1 << 20, room = (want + want / 4 + mib - 1) / mib * mib;
        if ((e = cudaMalloc((void **)&w.p, room)) != cudaSuccess) {
            cudaGetLastError();
            w.p = nullptr;
            return OP_WS_MEMORY;
        }
        if ((e = cudaMemsetAsync(w.p, 0, 256, stream)) != cudaSuccess) {
            cudaFree(w.p);
            w.p = nullptr;
            return OP_WS_CUDA;
        }
        w.bytes = room;
    } else if (w.recorded && w.stream != stream) {
        if ((e = cudaStreamWaitEvent(stream, w.ev, 0)) != cudaSuccess) return OP_WS_CUDA;
    }
    w.stream = stream;
    return OP_WS_OK;
}

// Behind the last launch of a call that used the workspace.
inline cudaError_t op_workspace_leave(OpWorkspace &w, cudaStream_t stream)
{
    if (w.capturing) return cudaSuccess;
    const cudaError_t e = cudaEventRecord(w.ev, stream);
    if (e == cudaSuccess) w.recorded = true;
    return e;
}

// A call's use of the workspace: left at the end of the call however it ends, so that what it has launched by then is
// waited for.
struct OpWorkspaceUse {
    OpWorkspace *w = nullptr;
    cudaStream_t stream = nullptr;
    OpWorkspaceUse() = default;
    OpWorkspaceUse(const OpWorkspaceUse &) = delete;
    OpWorkspaceUse &operator=(const OpWorkspaceUse &) = delete;
    ~OpWorkspaceUse()
    {
        if (w) op_workspace_leave(*w, stream);
    }
};

inline OpWorkspaceStatus op_workspace_take(OpWorkspace &w, size_t want, cudaStream_t stream, cudaError_t &e, OpWorkspaceUse &use)
{
    const OpWorkspaceStatus s = op_workspace_take(w, want, stream, e);
    if (s == OP_WS_OK) {
        use.w = &w;
        use.stream = stream;
    }
    return s;
}

inline cudaError_t op_workspace_leave(OpWorkspaceUse &use)
{
    if (!use.w) return cudaSuccess;
    OpWorkspace &w = *use.w;
    use.w = nullptr;
    return op_workspace_leave(w, use.stream);
}

inline void op_workspace_destroy(OpWorkspace &w)
{
    for (char *p : w.kept) cudaFree(p);
    if (w.p) cudaFree(w.p);
    if (w.ev) cudaEventDestroy(w.ev);
    w = OpWorkspace();
}
