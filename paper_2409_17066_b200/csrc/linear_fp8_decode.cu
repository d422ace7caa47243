// out = x W^T for at most 16 tokens over an e4m3 weight with 128 x 128 block scales.
//
// A CTA owns 16 * RG output rows; its warps take the 128-column blocks in turn (warp w blocks w, w + W, ...: neighbouring warps read
// neighbouring 128-byte lines of a row), with the next block's weights and activations in flight while one is multiplied
// (fp8_mma.cuh).  16-bit activations are quantized on the way, by the same rule as vptq_fp8_quantize: the four lanes that hold a
// token's block find its maximum with two shuffles.  The warps' sums meet in shared memory and are added in warp order, so a result
// does not depend on timing.
// Bound by HBM: M * N bytes.
#include "fp8_mma.cuh"

namespace vptq {

namespace {

template <int DT, bool VEC, int NG, int RG, int W>
__global__ void __launch_bounds__(32 * W)
linear_fp8_decode_kernel(const __grid_constant__ Fp8Linear P)
{
    __shared__ float part[W][NG * 8][RG * 16 + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int m0 = blockIdx.x * (16 * RG);
    const long long pitch = (P.N + 15ll) / 16 * 16;
    const int kbs = (P.N + FP8_BLOCK - 1) / FP8_BLOCK;
    const int cols = DT == VPTQ_DTYPE_E4M3 ? (int)pitch : P.N;

    const uint8_t *wrow[RG][2];
    const float *wscale[RG];
#pragma unroll
    for (int r = 0; r < RG; r++) {
#pragma unroll
        for (int h = 0; h < 2; h++) wrow[r][h] = P.w + min(m0 + 16 * r + 8 * h + g, P.M - 1) * pitch + 16 * t;
        wscale[r] = P.w_scale + (long long)(min(m0 + 16 * r, P.M - 1) / FP8_BLOCK) * kbs;
    }
    const uint8_t *xrow[NG];
    const float *xscale[NG];
#pragma unroll
    for (int n = 0; n < NG; n++) {
        const int token = 8 * n + g;
        xrow[n] = token < P.B ? reinterpret_cast<const uint8_t *>(P.x) + (DT == VPTQ_DTYPE_E4M3 ? token * pitch : (long long)token * P.N * 2) : nullptr;
        xscale[n] = DT == VPTQ_DTYPE_E4M3 ? P.x_scale + (long long)(token < P.B ? token : 0) * kbs : nullptr;
    }

    float acc[RG][NG][4] = {};
    WeightFrag a[RG];
    TokenRaw<DT, VEC> x[NG];
    float ws[RG];
    int kb = warp;
    auto fetch_weights = [&](int k) {
#pragma unroll
        for (int r = 0; r < RG; r++) {
            a[r] = load_weights(wrow[r][0] + (long long)k * FP8_BLOCK, wrow[r][1] + (long long)k * FP8_BLOCK, 0, pitch - 16 * t - (long long)k * FP8_BLOCK);
            ws[r] = __ldg(wscale[r] + k);
        }
    };
    auto fetch_tokens = [&](int k) {
#pragma unroll
        for (int n = 0; n < NG; n++) x[n] = load_token<DT, VEC>(xrow[n], xscale[n], k, t, cols);
    };
    if (kb < kbs) fetch_weights(kb);
    pdl_launch_dependents();
    pdl_wait();                                           // the activations may be the preceding kernel's
    if (kb < kbs) fetch_tokens(kb);
    for (; kb < kbs; kb += W) {
        WeightFrag ca[RG];
        float cs[RG];
        TokenRaw<DT, VEC> cx[NG];
#pragma unroll
        for (int r = 0; r < RG; r++) { ca[r] = a[r]; cs[r] = ws[r]; }
#pragma unroll
        for (int n = 0; n < NG; n++) cx[n] = x[n];
        if (kb + W < kbs) {
            fetch_weights(kb + W);
            fetch_tokens(kb + W);
        }
#pragma unroll
        for (int n = 0; n < NG; n++) {
            const TokenFrag b = quantize_token<DT, VEC>(cx[n]);
            const float2 s = scales_of_columns(b.scale, t);
#pragma unroll
            for (int r = 0; r < RG; r++) block_product(acc[r][n], ca[r], b, s.x * cs[r], s.y * cs[r]);
        }
    }
#pragma unroll
    for (int r = 0; r < RG; r++)
#pragma unroll
        for (int n = 0; n < NG; n++) {
            part[warp][8 * n + 2 * t][16 * r + g] = acc[r][n][0];
            part[warp][8 * n + 2 * t + 1][16 * r + g] = acc[r][n][1];
            part[warp][8 * n + 2 * t][16 * r + g + 8] = acc[r][n][2];
            part[warp][8 * n + 2 * t + 1][16 * r + g + 8] = acc[r][n][3];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < NG * 8 * RG * 16; i += 32 * W) {
        const int token = i / (RG * 16), row = i % (RG * 16);
        if (token >= P.B || m0 + row >= P.M) continue;
        float sum = part[0][token][row];
#pragma unroll
        for (int w = 1; w < W; w++) sum += part[w][token][row];
        store_out(P.out, (long long)token * P.M + m0 + row, sum, P.out_dtype);
    }
}

template <int DT, bool VEC, int NG, int RG, int W>
cudaError_t run(const Fp8Linear &P, cudaStream_t st)
{
    return launch_dependent("linear_fp8", linear_fp8_decode_kernel<DT, VEC, NG, RG, W>, ceil_div(P.M, 16 * RG), 32 * W, 0, st, P);
}

template <int DT, bool VEC>
cudaError_t choose(const Fp8Linear &P, cudaStream_t st)
{
    if (P.B <= 8) return run<DT, VEC, 1, 1, 8>(P, st);
    return run<DT, VEC, 2, 1, 8>(P, st);
}

}  // namespace

cudaError_t launch_linear_fp8_decode(const Fp8Linear &P, cudaStream_t st)
{
    const bool vec = P.N % 8 == 0;
    switch (P.x_dtype) {
    case VPTQ_DTYPE_E4M3: return choose<VPTQ_DTYPE_E4M3, true>(P, st);
    case VPTQ_DTYPE_BF16: return vec ? choose<VPTQ_DTYPE_BF16, true>(P, st) : choose<VPTQ_DTYPE_BF16, false>(P, st);
    default: return vec ? choose<VPTQ_DTYPE_FP16, true>(P, st) : choose<VPTQ_DTYPE_FP16, false>(P, st);
    }
}

}  // namespace vptq
