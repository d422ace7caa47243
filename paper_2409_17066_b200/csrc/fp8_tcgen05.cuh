// The product over e4m3 operands on the tensor cores (linear_fp8_tcgen05.cu).
#pragma once
#include "fp8.cuh"

namespace vptq {

// P.x in e4m3 with scales; *status is cleared, and set when a bounded wait gave up
cudaError_t launch_linear_fp8_tcgen05(const Fp8Linear &P, int *status, cudaStream_t st);

}  // namespace vptq
