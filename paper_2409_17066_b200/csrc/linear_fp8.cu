// vptq_linear_fp8: which kernels a call takes.
#include "fp8.cuh"
#include "fp8_tcgen05.cuh"

namespace vptq {

namespace {

bool decodes(int B) { return B <= FP8_DECODE_MAX_B; }
// 16-bit activations are quantized by a kernel of their own; the decode kernel does it itself
bool quantizes_before(int B, int x_dtype) { return x_dtype != VPTQ_DTYPE_E4M3 && !decodes(B); }

// workspace of the tensor-core kernel: the status word, then the activations' scales and e4m3 values
struct Workspace { long long scales, values, bytes; };
Workspace workspace_of(int N, int B, int x_dtype)
{
    Workspace w = {256, 256, decodes(B) ? 0 : 256};
    if (quantizes_before(B, x_dtype)) {
        w.values = w.scales + (4ll * B * ceil_div(N, FP8_BLOCK) + 255) / 256 * 256;
        w.bytes = w.values + B * fp8_row_bytes(N);
    }
    return w;
}

}  // namespace

long long linear_fp8_workspace_bytes(int N, int B, int x_dtype) { return workspace_of(N, B, x_dtype).bytes; }
int linear_fp8_launches(int B, int x_dtype) { return quantizes_before(B, x_dtype) ? 2 : 1; }
const char *linear_fp8_path(int B) { return decodes(B) ? "fp8_decode" : "fp8_tcgen05"; }

cudaError_t launch_linear_fp8(const Fp8Linear &P, void *ws, cudaStream_t st)
{
    uint8_t *w8 = reinterpret_cast<uint8_t *>(ws);
    Fp8Linear Q = P;
    if (quantizes_before(P.B, P.x_dtype)) {
        const Workspace w = workspace_of(P.N, P.B, P.x_dtype);
        const cudaError_t e = launch_fp8_quantize(P.x, P.x_dtype, P.B, P.N, P.N, 1, w8 + w.values, reinterpret_cast<float *>(w8 + w.scales), true, st);
        if (e != cudaSuccess) return e;
        Q.x = w8 + w.values;
        Q.x_scale = reinterpret_cast<const float *>(w8 + w.scales);
        Q.x_dtype = VPTQ_DTYPE_E4M3;
    }
    return decodes(P.B) ? launch_linear_fp8_decode(Q, st) : launch_linear_fp8_tcgen05(Q, reinterpret_cast<int *>(ws), st);
}

}  // namespace vptq
