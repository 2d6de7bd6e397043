#include "adapter_kernels.cuh"

namespace cs {
template AdapterKernel row_kernel<__nv_bfloat16>(const RowShape &);
template AdapterKernel wgrad_kernel<__nv_bfloat16>(int, int, int &);
}  // namespace cs
