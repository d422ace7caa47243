// vptq_linear_fp4: which kernels a call takes.
#include "fp4.cuh"
#include "fp4_tcgen05.cuh"

namespace vptq {

namespace {

bool few(int B) { return B <= FP4_FEW_MAX_B; }
// 16-bit activations are quantized by a kernel of their own; that for few tokens may do it itself
bool quantizes_before(int M, int B, int x_dtype) { return x_dtype != VPTQ_DTYPE_E2M1 && !(few(B) && linear_fp4_few_quantizes(M, B)); }

// workspace: the status word, then the activations' scales and e2m1 codes
struct Workspace { long long scales, values, bytes; };
Workspace workspace_of(int M, int N, int B, int x_dtype)
{
    Workspace w = {256, 256, 256};
    if (quantizes_before(M, B, x_dtype)) {
        w.values = w.scales + (fp4_scale_bytes(B, N) + 255) / 256 * 256;
        w.bytes = w.values + B * fp4_row_bytes(N);
    }
    return w;
}

}  // namespace

long long linear_fp4_workspace_bytes(int M, int N, int B, int x_dtype) { return workspace_of(M, N, B, x_dtype).bytes; }
int linear_fp4_launches(int M, int B, int x_dtype) { return quantizes_before(M, B, x_dtype) ? 2 : 1; }
const char *linear_fp4_path(int B) { return few(B) ? "fp4_few" : "fp4_tcgen05"; }

cudaError_t launch_linear_fp4(const Fp4Linear &P, void *ws, cudaStream_t st)
{
    uint8_t *w8 = reinterpret_cast<uint8_t *>(ws);
    Fp4Linear Q = P;
    if (quantizes_before(P.M, P.B, P.x_dtype)) {
        const Workspace w = workspace_of(P.M, P.N, P.B, P.x_dtype);
        const cudaError_t e = launch_fp4_quantize(P.x, P.x_dtype, P.B, P.N, P.N, w8 + w.values, w8 + w.scales, true, st);
        if (e != cudaSuccess) return e;
        Q.x = w8 + w.values;
        Q.x_scale = w8 + w.scales;
        Q.x_dtype = VPTQ_DTYPE_E2M1;
    }
    return few(P.B) ? launch_linear_fp4_few(Q, reinterpret_cast<int *>(ws), st) : launch_linear_fp4_tcgen05(Q, reinterpret_cast<int *>(ws), st);
}

}  // namespace vptq
