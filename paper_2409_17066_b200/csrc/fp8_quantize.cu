// Quantization to e4m3 with a scale per block: a = max(|x|) over the block (at least 2^-100), scale = a / 448 and r = 448 / a, each
// rounded to FP32, q = e4m3(x * r) with the product rounded to FP32 first; ties to even both times.  Multiplying by r and not
// dividing by the scale is the definition: one division a block, and a result that does not depend on how a division is formed.
//
// rows form (activations, a scale per 128 columns of a row): 16 lanes take the 128 columns of a block, eight adjacent ones each (a
// 16-byte load of 16-bit values, an 8-byte store); the block's maximum is four shuffles.  A half warp has UNROLL blocks in flight.
// blocks form (weights, a scale per 128 x 128): a CTA takes a block, 16 lanes a row of it, the values stay in registers between the
// maximum and the rounding: one pass over the matrix.
// 2 or 4 bytes read and one written a value: the blocks form is bound by HBM (28672 x 8192 from 16 bits 114 to 116 us, 6.1 TB/s; from FP32
// 168, 7.0 TB/s, four of five bytes of it read), the rows form by neither HBM nor its issue slots (63 % busy) alone: for eight values a lane it does
// four shuffles and both divisions, and four CTAs an SM have room for their registers (4096 x 8192 from 16 bits 25.3 us, 4.0 TB/s; from FP32
// 30.8, 5.4 TB/s).
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
    long long step;            // rows form: blocks that all half warps take at a time, and the same as rows and column blocks
    int step_rows, step_cols;
};

template <int DT, bool VEC, int UNROLL>
__global__ void __launch_bounds__(THREADS)
quantize_rows_kernel(const __grid_constant__ QuantizeParams P)
{
    if (P.early) pdl_launch_dependents();
    pdl_wait();
    // blocks of the matrix, rows after one another, are dealt out over the half warps; row and column block are counted on without divisions
    const int lane = threadIdx.x & 15, half = (threadIdx.x >> 4) & 1;
    const long long first = ((long long)blockIdx.x * THREADS + threadIdx.x) >> 4;
    int row = (int)(first / P.col_blocks), cb = (int)(first % P.col_blocks);
    // (a warp's two halves run the same number of rounds: shuffles)
    const long long n = (long long)P.rows * P.col_blocks;
    for (long long b0 = first - half; b0 < n; b0 += P.step * UNROLL) {
        Eight<DT, VEC> e[UNROLL];
        int rows[UNROLL], cols[UNROLL];
        uint32_t m[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; u++) {
            rows[u] = row; cols[u] = cb * FP8_BLOCK + lane * 8;
            e[u] = load_eight<DT, VEC>(reinterpret_cast<const uint8_t *>(P.x) + (row < P.rows ? row : 0) * P.ld * Act<DT>::BYTES, row < P.rows ? cols[u] : P.cols, P.cols);
            cb += P.step_cols; row += P.step_rows;
            if (cb >= P.col_blocks) { cb -= P.col_blocks; row++; }
        }
#pragma unroll
        for (int u = 0; u < UNROLL; u++) {
            m[u] = magnitude(e[u]);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) m[u] = max(m[u], __shfl_xor_sync(0xffffffffu, m[u], o));
        }
#pragma unroll
        for (int u = 0; u < UNROLL; u++) {
            if (rows[u] >= P.rows) continue;
            const Fp8Scale s = fp8_scale(__uint_as_float(m[u]));
            store_eight(P.q + rows[u] * P.pitch, P.pitch, cols[u], P.cols, e[u], s.factor);
            if (lane == 0) P.scale[(long long)rows[u] * P.col_blocks + cols[u] / FP8_BLOCK] = s.scale;
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
    Eight<DT, VEC> v[ROUNDS];
#pragma unroll
    for (int i = 0; i < ROUNDS; i++) {
        const long long row = (long long)rb * FP8_BLOCK + i * ROWS + r0;
        v[i] = load_eight<DT, VEC>(reinterpret_cast<const uint8_t *>(P.x) + (row < P.rows ? row : 0) * P.ld * Act<DT>::BYTES, row < P.rows ? c : P.cols, P.cols);
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < ROUNDS; i++) m = max(m, magnitude(v[i]));
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
        store_eight(P.q + row * P.pitch, P.pitch, c, P.cols, v[i], s.factor);
    }
}

template <int DT, bool VEC, int UNROLL>
cudaError_t launch_rows(QuantizeParams P, long long ctas, cudaStream_t st)
{
    P.step = ctas * (THREADS / 16);
    P.step_rows = (int)(P.step / P.col_blocks);
    P.step_cols = (int)(P.step % P.col_blocks);
    return launch_dependent("fp8_quantize", quantize_rows_kernel<DT, VEC, UNROLL>, (int)ctas, THREADS, 0, st, P);
}

template <int DT, bool VEC>
cudaError_t launch(const QuantizeParams &P, int block_rows, cudaStream_t st)
{
    if (block_rows != 1) {
        const long long blocks = (long long)ceil_div(P.rows, FP8_BLOCK) * P.col_blocks;
        quantize_blocks_kernel<DT, VEC><<<(unsigned)blocks, THREADS, 0, st>>>(P);
        return cudaGetLastError();
    }
    // small calls: a block of values per half warp; large ones: four in flight, on eight CTAs an SM, of which four (FP32: three) run at a time
    const long long n = (long long)P.rows * P.col_blocks, per_cta = THREADS / 16;
    const long long resident = (long long)device_sm_count() * 8;
    const long long ctas = (n + per_cta - 1) / per_cta;
    if (ctas <= resident) return launch_rows<DT, VEC, 1>(P, ctas, st);
    return launch_rows<DT, VEC, 4>(P, (ctas + 3) / 4 < resident ? (ctas + 3) / 4 : resident, st);
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
