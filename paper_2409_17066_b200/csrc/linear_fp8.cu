// vptq_linear_fp8: which kernels a call takes.
#include "fp8.cuh"

namespace vptq {

long long linear_fp8_workspace_bytes(int M, int N, int B, int x_dtype) { return 0; }
int linear_fp8_launches(int M, int N, int B, int x_dtype) { return ceil_div(B, FP8_DECODE_MAX_B); }
const char *linear_fp8_path(int M, int N, int B, int x_dtype) { return "fp8_decode"; }

cudaError_t launch_linear_fp8(const Fp8Linear &P, void *ws, cudaStream_t st)
{
    const long long x_row = P.x_dtype == VPTQ_DTYPE_E4M3 ? fp8_row_bytes(P.N) : 2ll * P.N, out_row = (P.out_dtype == VPTQ_DTYPE_FP32 ? 4ll : 2ll) * P.M;
    for (int b = 0; b < P.B; b += FP8_DECODE_MAX_B) {
        Fp8Linear Q = P;
        Q.B = P.B - b < FP8_DECODE_MAX_B ? P.B - b : FP8_DECODE_MAX_B;
        Q.x = reinterpret_cast<const uint8_t *>(P.x) + b * x_row;
        if (P.x_scale != nullptr) Q.x_scale = P.x_scale + (long long)b * ceil_div(P.N, FP8_BLOCK);
        Q.out = reinterpret_cast<uint8_t *>(P.out) + b * out_row;
        const cudaError_t e = launch_linear_fp8_decode(Q, st);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace vptq
