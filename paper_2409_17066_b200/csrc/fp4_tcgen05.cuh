// The product over e2m1 operands: on tcgen05 (linear_fp4_tcgen05.cu), and for a few tokens (linear_fp4_few.cu).
#pragma once
#include "fp4.cuh"

namespace vptq {

// P.x in e2m1 with scales, early: by the kernel launched just before (Behind::THEN); *status is cleared, and set when a bounded wait gave up
cudaError_t launch_linear_fp4_tcgen05(const Fp4Linear &P, int *status, bool early, cudaStream_t st);

// a few tokens in 16 bits over a small weight, quantized on the way; no status word
bool linear_fp4_few_takes(int M, int N, int B, int x_dtype);
cudaError_t launch_linear_fp4_few(const Fp4Linear &P, cudaStream_t st);

}  // namespace vptq
