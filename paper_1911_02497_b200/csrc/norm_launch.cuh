// Between the host side of the norm and the source files that compile its kernels for a type.
#pragma once
#include "norm.cuh"
#include "op_args.h"

// How a backward call is cut: CTAs, and the slots of sums for dgain that they leave.
struct NormBackPlan {
    int grid, slots;
};

// `access`: values that all operands allow at once. backward: `run` false only fills the plan.
template <class T> int norm_forward_launch(condensa_ctx *ctx, const cs::NormParams &P, int access, cudaStream_t stream);
template <class T> int norm_backward_launch(condensa_ctx *ctx, const cs::NormBackParams &P, NormBackPlan &plan, int access, bool run, cudaStream_t stream);
