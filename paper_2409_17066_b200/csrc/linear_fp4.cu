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

// Loads of the weight may go ahead of the tokens' quantization only if the product is let in when all before that has ended, not at once: worth it
// where the loads take longer than the wait, and with some tokens, whose quantization takes longer too.  Gains over weights of 2560 to 11008 columns, in a
// graph / call by call, weights one after the other out of HBM:
//   9 to 48 tokens:  14 MB -7 % / +2 %, 35 MB -4 / +1, 58 MB -4 / +1, 72 MB -3 / +3, 96 MB +1 / +4
//   96 to 700:       14 MB -1 % / +3 %, 21 MB 0 / +3, 35 MB +1 / +3, 58 MB +1 / +3, 96 MB +1 / +3
// and with one weight that stays in L2
//   9 to 48:         35 MB -6 % / -4 %, 58 MB -2 / -1, 72 MB +2 / 0, 96 MB +2 / +4
//   96 to 700:       14 MB -5 % / 0 %, 25 MB -2 / +1, 35 MB -1 / 0, 58 MB +2 / +2, 96 MB +1 / +3
bool loads_early(long long weight_bytes, int tokens) { return weight_bytes >= (tokens < 96 ? 80 << 20 : 24 << 20); }

}  // namespace

long long linear_fp4_workspace_bytes(int M, int N, int B, int x_dtype) { return workspace_of(M, N, B, x_dtype).bytes; }
int linear_fp4_launches(int M, int N, int B, int x_dtype) { return x_dtype != VPTQ_DTYPE_E2M1 && !linear_fp4_few_takes(M, N, B, x_dtype) ? 2 : 1; }
const char *linear_fp4_path(int M, int N, int B, int x_dtype) { return linear_fp4_few_takes(M, N, B, x_dtype) ? "fp4_few" : "fp4_tcgen05"; }

cudaError_t launch_linear_fp4(const Fp4Linear &P, void *ws, cudaStream_t st)
{
    if (linear_fp4_few_takes(P.M, P.N, P.B, P.x_dtype)) return launch_linear_fp4_few(P, st);
    uint8_t *w8 = reinterpret_cast<uint8_t *>(ws);
    Fp4Linear Q = P;
    const bool early = P.x_dtype != VPTQ_DTYPE_E2M1 && loads_early(P.M * fp4_row_bytes(P.N), P.B);
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
