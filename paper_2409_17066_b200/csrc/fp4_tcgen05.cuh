// The product over e2m1 operands on the tensor cores (linear_fp4_tcgen05.cu).
#pragma once
#include "fp4.cuh"

namespace vptq {

// P.x in e2m1 with scales; *status is cleared, and set when a bounded wait gave up
cudaError_t launch_linear_fp4_tcgen05(const Fp4Linear &P, int *status, cudaStream_t st);

}  // namespace vptq
