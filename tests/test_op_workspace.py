"""The operators' workspace (csrc/op_workspace.h) against a fake of the CUDA runtime calls that it makes: which blocks live,
which work waits for which. No GPU needed."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

FAKE = r"""
#include "op_workspace.h"
#include <cstdio>
#include <cstdlib>
#include <set>
#include <string>

static std::set<void *> live;
static std::set<cudaStream_t> captured;
static bool no_memory = false;
static std::string log_;

cudaError_t cudaStreamIsCapturing(cudaStream_t s, cudaStreamCaptureStatus *st)
{
    *st = captured.count(s) ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone;
    return cudaSuccess;
}
cudaError_t cudaEventCreateWithFlags(cudaEvent_t *e, unsigned) { *e = (cudaEvent_t)0x99; return cudaSuccess; }
cudaError_t cudaEventDestroy(cudaEvent_t) { log_ += "destroy;"; return cudaSuccess; }
cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t s) { log_ += "record" + std::to_string((size_t)s) + ";"; return cudaSuccess; }
cudaError_t cudaStreamWaitEvent(cudaStream_t s, cudaEvent_t, unsigned) { log_ += "wait" + std::to_string((size_t)s) + ";"; return cudaSuccess; }
cudaError_t cudaDeviceSynchronize() { log_ += "sync;"; return cudaSuccess; }
cudaError_t cudaMemsetAsync(void *, int, size_t n, cudaStream_t) { log_ += "zero" + std::to_string(n) + ";"; return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaMalloc(void **p, size_t)
{
    if (no_memory) return cudaErrorMemoryAllocation;
    *p = malloc(16);
    live.insert(*p);
    return cudaSuccess;
}
cudaError_t cudaFree(void *p) { if (!live.erase(p)) log_ += "twice;"; return cudaSuccess; }

static const cudaStream_t A = (cudaStream_t)1, B = (cudaStream_t)2;
static cudaError_t e = cudaSuccess;
#define CHECK(c) do { if (!(c)) { printf("line %d: %s [%s]\n", __LINE__, #c, log_.c_str()); exit(1); } } while (0)
"""


@pytest.fixture()
def run(tmp_path):
    def run(body):
        src, exe = str(tmp_path / "t.cpp"), str(tmp_path / "t")
        open(src, "w").write(FAKE + "int main() { OpWorkspace w;\n" + body + "\nreturn 0; }\n")
        subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-Wno-unused", "-I", os.path.join(ROOT, "paper_1911_02497_b200", "csrc"),
                        "-I", "/usr/local/cuda/include", "-o", exe, src], check=True)
        r = subprocess.run([exe], capture_output=True, text=True)
        assert r.returncode == 0, r.stdout
    return run


def test_a_block_that_a_capture_has_seen_outlives_a_growth(run):
    """A graph keeps the addresses of the block that it was captured with, so a replay after a larger call needs that block."""
    run(r"""
        CHECK(op_workspace_take(w, 1000, A, e) == OP_WS_OK && op_workspace_leave(w, A) == cudaSuccess);
        void *first = w.p;
        captured.insert(A);
        CHECK(op_workspace_take(w, 1000, A, e) == OP_WS_OK && w.p == first && op_workspace_leave(w, A) == cudaSuccess);
        captured.clear();
        CHECK(op_workspace_take(w, 64 << 20, A, e) == OP_WS_OK && w.p != first);
        CHECK(live.count(first) && live.size() == 2);
        // the larger block has been in no capture: it goes when it is outgrown
        void *second = w.p;
        CHECK(op_workspace_take(w, 512 << 20, A, e) == OP_WS_OK);
        CHECK(live.count(first) && !live.count(second) && live.size() == 2);
        op_workspace_destroy(w);
        CHECK(live.empty() && log_.find("twice") == std::string::npos);
        op_workspace_destroy(w);
        CHECK(log_.find("twice") == std::string::npos);
    """)


def test_a_block_survives_a_growth_that_fails(run):
    run(r"""
        CHECK(op_workspace_take(w, 1000, A, e) == OP_WS_OK);
        void *first = w.p;
        captured.insert(A);
        CHECK(op_workspace_take(w, 1000, A, e) == OP_WS_OK);
        captured.clear();
        no_memory = true;
        CHECK(op_workspace_take(w, 64 << 20, A, e) == OP_WS_MEMORY && e == cudaErrorMemoryAllocation);
        no_memory = false;
        CHECK(live.count(first));
        CHECK(op_workspace_take(w, 64 << 20, A, e) == OP_WS_OK && live.size() == 2);
        op_workspace_destroy(w);
        CHECK(live.empty());
    """)


def test_blocks_that_no_graph_knows_go_when_they_are_outgrown(run):
    run(r"""
        for (size_t n = 1 << 20; n <= (size_t)1 << 30; n *= 4) {
            CHECK(op_workspace_take(w, n, A, e) == OP_WS_OK && op_workspace_leave(w, A) == cudaSuccess);
            CHECK(live.size() == 1);
        }
        op_workspace_destroy(w);
        CHECK(live.empty());
    """)


def test_calls_are_ordered_across_streams_and_captures_are_not(run):
    run(r"""
        CHECK(op_workspace_take(w, 1000, A, e) == OP_WS_OK && log_ == "sync;zero256;" && op_workspace_leave(w, A) == cudaSuccess);
        log_ = "";
        CHECK(op_workspace_take(w, 1000, A, e) == OP_WS_OK && log_ == "" && op_workspace_leave(w, A) == cudaSuccess && log_ == "record1;");
        log_ = "";
        CHECK(op_workspace_take(w, 1000, B, e) == OP_WS_OK && log_ == "wait2;" && op_workspace_leave(w, B) == cudaSuccess);
        captured.insert(A);
        log_ = "";
        CHECK(op_workspace_take(w, 1000, A, e) == OP_WS_OK && op_workspace_leave(w, A) == cudaSuccess && log_ == "");
        CHECK(op_workspace_take(w, 64 << 20, A, e) == OP_WS_CAPTURE && log_ == "");
        op_workspace_destroy(w);
    """)


def test_a_call_that_fails_midway_is_still_ordered(run):
    """Whatever a call has launched by then uses the block: the next call on another stream waits for it."""
    run(r"""
        {
            OpWorkspaceUse use;
            CHECK(op_workspace_take(w, 1000, A, e, use) == OP_WS_OK);
        }                                   // an error return between the launches
        CHECK(log_ == "sync;zero256;record1;" && w.recorded);
        log_ = "";
        {
            OpWorkspaceUse use;
            CHECK(op_workspace_take(w, 1000, B, e, use) == OP_WS_OK && log_ == "wait2;");
            CHECK(op_workspace_leave(use) == cudaSuccess && log_ == "wait2;record2;");
        }
        CHECK(log_ == "wait2;record2;");    // once
        log_ = "";
        {
            OpWorkspaceUse use;             // a call that needs no workspace
            CHECK(op_workspace_leave(use) == cudaSuccess);
        }
        captured.insert(A);
        {
            OpWorkspaceUse use;
            CHECK(op_workspace_take(w, 1000, A, e, use) == OP_WS_OK);
            CHECK(op_workspace_take(w, 64 << 20, A, e, use) == OP_WS_CAPTURE);
        }
        CHECK(log_ == "");
        op_workspace_destroy(w);
    """)
