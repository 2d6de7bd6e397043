// Launches of the adapter kernels. Their instances are compiled per type, side by side (adapter_bf16.cu, _f16.cu, _f32.cu).
#pragma once
#include "adapter.cuh"
#include "ctx.cuh"

namespace cs {

// A kernel instance: its function, shared memory, and how many CTAs an SM holds.
struct AdapterKernel {
    const void *f;
    int smem, per_sm, threads;
};

// Shape of the row kernel's instances: by tile height, largest rank, access width.
struct RowShape {
    int tm, rank, vec;
};

template <class T> AdapterKernel row_kernel(const RowShape &s);
template <class T> AdapterKernel wgrad_kernel(int rank, int vec, int &strip);

extern template AdapterKernel row_kernel<__nv_bfloat16>(const RowShape &);
extern template AdapterKernel row_kernel<__half>(const RowShape &);
extern template AdapterKernel row_kernel<float>(const RowShape &);
extern template AdapterKernel wgrad_kernel<__nv_bfloat16>(int, int, int &);
extern template AdapterKernel wgrad_kernel<__half>(int, int, int &);
extern template AdapterKernel wgrad_kernel<float>(int, int, int &);

}  // namespace cs
