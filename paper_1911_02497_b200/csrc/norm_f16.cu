#include "norm_kernels.cuh"

template int norm_forward_launch<__half>(condensa_ctx *, const cs::NormParams &, int, cudaStream_t);
template int norm_backward_launch<__half>(condensa_ctx *, const cs::NormBackParams &, NormBackPlan &, int, bool, cudaStream_t);
