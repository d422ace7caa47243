// vptq_linear_fp4: which kernels a call takes.
#include "fp4.cuh"
#include "fp4_tcgen05.cuh"

namespace vptq {

namespace {

// workspace of the tensor-core kernel: the status word, then the scales and e2m1 codes of 16-bit activations, which a kernel in front of it makes
struct Workspace { long long scales, values, bytes; };
Workspace workspace_of(int M, int N, int B, int x_dtype)
{
    Workspace w = {256, 256, linear_fp4_few_takes(M, N, B, x_dtype) ? 0 : 256};
    if (w.bytes > 0 && x_dtype != VPTQ_DTYPE_E2M1) {
        w.values = w.scales + (fp4_scale_bytes(B, N) + 255) / 256 * 256;
        w.bytes = w.values + B * fp4_row_bytes(N);
    }
    return w;
}

}  // namespace

long long linear_fp4_workspace_bytes(int M, int N, int B, int x_dtype) { return workspace_of(M, N, B, x_dtype).bytes; }
int linear_fp4_launches(int M, int N, int B, int x_dtype) { return x_dtype != VPTQ_DTYPE_E2M1 && !linear_fp4_few_takes(M, N, B, x_dtype) ? 2 : 1; }
const char *linear_fp4_path(int M, int N, int B, int x_dtype) { return linear_fp4_few_takes(M, N, B, x_dtype) ? "fp4_few" : "fp4_tcgen05"; }

cudaError_t launch_linear_fp4(const Fp4Linear &P, void *ws, cudaStream_t st)
{
    if (linear_fp4_few_takes(P.M, P.N, P.B, P.x_dtype)) return launch_linear_fp4_few(P, st);
    uint8_t *w8 = reinterpret_cast<uint8_t *>(ws);
    Fp4Linear Q = P;
    // Loads of the weight may go ahead of the tokens' quantization only if the product is let in when all before that has ended, not at once: worth it for
    // weights that come from HBM (one after the other, 28672 x 8192 at 16 tokens 25.9 -> 24.6 us, 14336 x 4096 at 500 22.5 -> 21.5; still in L2 17.3 ->
    // 17.4), too late for small ones (in a graph 300 x 600 at 40 tokens 6.9 -> 7.9, 11008 x 4096 at 128 9.5 -> 10.0).
    const bool early = P.x_dtype != VPTQ_DTYPE_E2M1 && P.M * fp4_row_bytes(P.N) >= 28 << 20;
    if (P.x_dtype != VPTQ_DTYPE_E2M1) {
        const Workspace w = workspace_of(P.M, P.N, P.B, P.x_dtype);
        const cudaError_t e = launch_fp4_quantize(P.x, P.x_dtype, P.B, P.N, P.N, w8 + w.values, w8 + w.scales, early ? Behind::THEN : Behind::AT_ONCE, st);
        if (e != cudaSuccess) return e;
        Q.x = w8 + w.values;
        Q.x_scale = w8 + w.scales;
        Q.x_dtype = VPTQ_DTYPE_E2M1;
    }
    return launch_linear_fp4_tcgen05(Q, reinterpret_cast<int *>(ws), early, st);
}

}  // namespace vptq
