// The product over e2m1 operands on the tensor cores: linear_fp4_tcgen05.cu, and linear_fp4_few.cu for a few tokens.
#pragma once
#include "fp4.cuh"

namespace vptq {

// P.x in e2m1 with scales; *status is cleared, and set when a bounded wait gave up
cudaError_t launch_linear_fp4_tcgen05(const Fp4Linear &P, int *status, cudaStream_t st);

// P.x of any type
constexpr int FP4_FEW_MAX_B = 16;
bool linear_fp4_few_takes(int M, int N, int B);
cudaError_t launch_linear_fp4_few(const Fp4Linear &P, int *status, cudaStream_t st);

}  // namespace vptq
