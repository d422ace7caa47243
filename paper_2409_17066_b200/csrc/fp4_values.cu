// Values of an e2m1 matrix: code times its block's power of two, exact in FP32, rounded once to the result's type.
//
// A lane takes eight adjacent columns: four bytes of codes, one scale byte, a 16-byte store of 16-bit values; UNROLL rows of a tile at
// a time, so that as many reads are in flight.  17/32 of a byte read and 2 or 4 written a value: bound by HBM's writes.
#include "fp4.cuh"

namespace vptq {

namespace {

constexpr int THREADS = 256, UNROLL = 4, ROWS = THREADS / 16 * UNROLL;       // rows of a CTA, 128 columns wide

struct ValuesParams {
    const uint8_t *q, *scale;
    int rows, cols, col_tiles;
    long long pitch;
    void *out;
};

template <int DT, bool VEC>
__global__ void __launch_bounds__(THREADS)
fp4_values_kernel(const __grid_constant__ ValuesParams P)
{
    pdl_wait();
    const int lane = threadIdx.x & 15, sub = threadIdx.x >> 4;
    const int ct = (int)(blockIdx.x % P.col_tiles), row0 = (int)(blockIdx.x / P.col_tiles) * ROWS + sub, c = ct * FP4_TILE_COLS + lane * 8;
    if (c >= P.cols) return;
    uint32_t q[UNROLL], b[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; u++) {
        const int row = row0 + u * (THREADS / 16);
        if (row < P.rows) {
            q[u] = __ldcs(reinterpret_cast<const uint32_t *>(P.q + row * P.pitch + c / 2));
            b[u] = __ldg(P.scale + ((long long)(row / FP4_TILE_ROWS) * P.col_tiles + ct) * FP4_TILE_BYTES + fp4_scale_at(row % FP4_TILE_ROWS, lane >> 2));
        }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; u++) {
        const int row = row0 + u * (THREADS / 16);
        if (row >= P.rows) break;
        float v[8];
        fp4_scaled8(q[u], fp4_scale_value(b[u]), v);
        store_values8<DT, VEC>(reinterpret_cast<uint8_t *>(P.out) + (long long)row * P.cols * (DT == VPTQ_DTYPE_FP32 ? 4 : 2), c, P.cols, v);
    }
}

template <int DT>
cudaError_t launch(const ValuesParams &P, cudaStream_t st)
{
    const long long ctas = (long long)ceil_div(P.rows, ROWS) * P.col_tiles;
    if (P.cols % (DT == VPTQ_DTYPE_FP32 ? 4 : 8) == 0) return launch_dependent("fp4_values", fp4_values_kernel<DT, true>, (int)ctas, THREADS, 0, st, P);
    return launch_dependent("fp4_values", fp4_values_kernel<DT, false>, (int)ctas, THREADS, 0, st, P);
}

}  // namespace

cudaError_t launch_fp4_values(const uint8_t *q, const uint8_t *scale, int rows, int cols, int out_dtype, void *out, cudaStream_t st)
{
    ValuesParams P;
    P.q = q; P.scale = scale; P.rows = rows; P.cols = cols; P.col_tiles = ceil_div(cols, FP4_TILE_COLS);
    P.pitch = fp4_row_bytes(cols); P.out = out;
    switch (out_dtype) {
    case VPTQ_DTYPE_FP16: return launch<VPTQ_DTYPE_FP16>(P, st);
    case VPTQ_DTYPE_BF16: return launch<VPTQ_DTYPE_BF16>(P, st);
    default: return launch<VPTQ_DTYPE_FP32>(P, st);
    }
}

}  // namespace vptq
