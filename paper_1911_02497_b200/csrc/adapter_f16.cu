#include "adapter_kernels.cuh"

namespace cs {
template AdapterKernel row_kernel<__half>(const RowShape &);
template AdapterKernel wgrad_kernel<__half>(int, int, int &);
}  // namespace cs
