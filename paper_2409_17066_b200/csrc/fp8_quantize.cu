// Quantization to e4m3 with a scale per block: a = max(|x|) over the block (at least 2^-100), scale = a / 448 and r = 448 / a, each
// rounded to FP32, q = e4m3(x * r) with the product rounded to FP32 first; ties to even both times.  Multiplying by r and not
// dividing by the scale is the definition: one division a block, and a result that does not depend on how a division is formed.
//
// rows form (activations, a scale per 128 columns of a row): 16 lanes take the 128 columns of a block, eight adjacent ones each (a
// 16-byte load of 16-bit values, an 8-byte store); the block's maximum is four shuffles.  A half warp has UNROLL blocks in flight.
// blocks form (weights, a scale per 128 x 128): a CTA takes a block, 16 lanes a row of it, the values stay in registers between the
// maximum and the rounding: one pass over the matrix.
// Both are bound by HBM: 2 or 4 bytes read and one written a value.
#include "fp8.cuh"

namespace vptq {

namespace {

constexpr int THREADS = 256;

struct QuantizeParams {
    const void *x;
    int rows, cols;
    long long ld, pitch;
    int col_blocks;
    uint8_t *q;
    float *scale;
    int early;
};

// eight values at column c of a row of q: pad columns (zeros) are written up to the row's end
__device__ __forceinline__ void store_eight(uint8_t *row, long long pitch, int c, const float (&v)[8], float factor)
{
    if (c >= pitch) return;
    uint2 o;
    o.x = fp8_quad(v[0] * factor, v[1] * factor, v[2] * factor, v[3] * factor);
    o.y = fp8_quad(v[4] * factor, v[5] * factor, v[6] * factor, v[7] * factor);
    *reinterpret_cast<uint2 *>(row + c) = o;
}

// (a value beyond the row's end is 0, and 0 * factor is not when the factor is infinite or NaN: the pad bytes are zeros all the same)
__device__ __forceinline__ void clear_pad(uint8_t *row, long long pitch, int c, int cols)
{
    for (int i = max(c, cols); i < c + 8 && i < pitch; i++) row[i] = 0;
}

template <int DT, bool VEC, int UNROLL>
__global__ void __launch_bounds__(THREADS)
quantize_rows_kernel(const __grid_constant__ QuantizeParams P)
{
    if (P.early) pdl_launch_dependents();
    pdl_wait();
    const long long n = (long long)P.rows * P.col_blocks;
    const int lane = threadIdx.x & 15;
    const long long first = ((long long)blockIdx.x * THREADS + threadIdx.x) >> 4, step = ((long long)gridDim.x * THREADS) >> 4;
    // (a warp's two halves run the same number of rounds: shuffles)
    for (long long b0 = first; b0 - ((threadIdx.x >> 4) & 1) < n; b0 += step * UNROLL) {
        float v[UNROLL][8];
        uint32_t m[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; u++) {
            const long long b = b0 + u * step, row = b / P.col_blocks;
            const int c = (int)(b % P.col_blocks) * FP8_BLOCK + lane * 8;
            if (b < n) {
                load_values<DT, VEC, 8>(reinterpret_cast<const uint8_t *>(P.x) + row * P.ld * Act<DT>::BYTES, c, P.cols, v[u]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++) v[u][i] = 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < UNROLL; u++) {
            m[u] = magnitude<8>(v[u]);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) m[u] = max(m[u], __shfl_xor_sync(0xffffffffu, m[u], o));
        }
#pragma unroll
        for (int u = 0; u < UNROLL; u++) {
            const long long b = b0 + u * step, row = b / P.col_blocks;
            if (b >= n) continue;
            const int c = (int)(b % P.col_blocks) * FP8_BLOCK + lane * 8;
            const Fp8Scale s = fp8_scale(__uint_as_float(m[u]));
            store_eight(P.q + row * P.pitch, P.pitch, c, v[u], s.factor);
            if (c + 8 > P.cols) clear_pad(P.q + row * P.pitch, P.pitch, c, P.cols);
            if (lane == 0) P.scale[b] = s.scale;
        }
    }
}

template <int DT, bool VEC>
__global__ void __launch_bounds__(THREADS)
quantize_blocks_kernel(const __grid_constant__ QuantizeParams P)
{
    constexpr int ROWS = THREADS / 16, ROUNDS = FP8_BLOCK / ROWS;
    __shared__ uint32_t part[THREADS / 32];
    const int lane = threadIdx.x & 15, r0 = threadIdx.x >> 4;
    const int cb = blockIdx.x % P.col_blocks, rb = blockIdx.x / P.col_blocks;
    const int c = cb * FP8_BLOCK + lane * 8;
    float v[ROUNDS][8];
#pragma unroll
    for (int i = 0; i < ROUNDS; i++) {
        const long long row = (long long)rb * FP8_BLOCK + i * ROWS + r0;
        if (row < P.rows) {
            load_values<DT, VEC, 8>(reinterpret_cast<const uint8_t *>(P.x) + row * P.ld * Act<DT>::BYTES, c, P.cols, v[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) v[i][j] = 0.f;
        }
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < ROUNDS; i++) m = max(m, magnitude<8>(v[i]));
    m = __reduce_max_sync(0xffffffffu, m);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 32; i++) m = max(m, part[i]);
    const Fp8Scale s = fp8_scale(__uint_as_float(m));
    if (threadIdx.x == 0) P.scale[blockIdx.x] = s.scale;
#pragma unroll
    for (int i = 0; i < ROUNDS; i++) {
        const long long row = (long long)rb * FP8_BLOCK + i * ROWS + r0;
        if (row >= P.rows) break;
        store_eight(P.q + row * P.pitch, P.pitch, c, v[i], s.factor);
        if (c + 8 > P.cols) clear_pad(P.q + row * P.pitch, P.pitch, c, P.cols);
    }
}

template <int DT, bool VEC>
cudaError_t launch(const QuantizeParams &P, int block_rows, cudaStream_t st)
{
    if (block_rows != 1) {
        const long long blocks = (long long)ceil_div(P.rows, FP8_BLOCK) * P.col_blocks;
        quantize_blocks_kernel<DT, VEC><<<(unsigned)blocks, THREADS, 0, st>>>(P);
        return cudaGetLastError();
    }
    // small calls: a block of values per half warp; large ones: four in flight, and CTAs that stay
    const long long n = (long long)P.rows * P.col_blocks, per_cta = THREADS / 16;
    const long long resident = (long long)device_sm_count() * 8;
    const long long ctas = (n + per_cta - 1) / per_cta;
    if (ctas <= resident) return launch_dependent("fp8_quantize", quantize_rows_kernel<DT, VEC, 1>, (int)ctas, THREADS, 0, st, P);
    const long long want = (ctas + 3) / 4;
    return launch_dependent("fp8_quantize", quantize_rows_kernel<DT, VEC, 4>, (int)(want < resident ? want : resident), THREADS, 0, st, P);
}

}  // namespace

cudaError_t launch_fp8_quantize(const void *x, int x_dtype, int rows, int cols, long long ld, int block_rows, uint8_t *q, float *scale,
                                bool early, cudaStream_t st)
{
    QuantizeParams P;
    P.x = x; P.rows = rows; P.cols = cols; P.ld = ld; P.pitch = fp8_row_bytes(cols);
    P.col_blocks = ceil_div(cols, FP8_BLOCK);
    P.q = q; P.scale = scale; P.early = early ? 1 : 0;
    const int bytes = x_dtype == VPTQ_DTYPE_FP32 ? 4 : 2, per = 16 / bytes;
    const bool vec = (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && cols % per == 0 && (rows == 1 || ld % per == 0);
    switch (x_dtype) {
    case VPTQ_DTYPE_FP16: return vec ? launch<VPTQ_DTYPE_FP16, true>(P, block_rows, st) : launch<VPTQ_DTYPE_FP16, false>(P, block_rows, st);
    case VPTQ_DTYPE_BF16: return vec ? launch<VPTQ_DTYPE_BF16, true>(P, block_rows, st) : launch<VPTQ_DTYPE_BF16, false>(P, block_rows, st);
    default: return vec ? launch<VPTQ_DTYPE_FP32, true>(P, block_rows, st) : launch<VPTQ_DTYPE_FP32, false>(P, block_rows, st);
    }
}

}  // namespace vptq
