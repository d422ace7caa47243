// The product over e2m1 operands: on tcgen05 (linear_fp4_tcgen05.cu), and for a few tokens (linear_fp4_few.cu).
#pragma once
#include "fp4.cuh"

namespace vptq {

// P.x in e2m1 with scales; *status is cleared, and set when a bounded wait gave up
cudaError_t launch_linear_fp4_tcgen05(const Fp4Linear &P, int *status, cudaStream_t st);

// at most FP4_FEW_MAX_B tokens, in e2m1 or, where it quantizes them itself, in 16 bits
constexpr int FP4_FEW_MAX_B = 16;
bool linear_fp4_few_quantizes(int M, int B);
cudaError_t launch_linear_fp4_few(const Fp4Linear &P, int *status, cudaStream_t st);

}  // namespace vptq
