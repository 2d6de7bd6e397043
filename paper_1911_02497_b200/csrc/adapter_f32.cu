#include "adapter_kernels.cuh"

namespace cs {
template AdapterKernel row_kernel<float>(const RowShape &);
template AdapterKernel wgrad_kernel<float>(int, int, int &);
}  // namespace cs
