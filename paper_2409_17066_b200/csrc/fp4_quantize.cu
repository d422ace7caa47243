// Quantization to e2m1 with a power of two for every 32 columns of a row: the block's largest magnitude gives the scale by one integer
// addition (fp4.cuh), the codes are the hardware's conversion of x / scale, which is exact before it is rounded.
//
// 16 lanes take 128 columns of a row, eight adjacent values each (a 16-byte load of 16-bit values, a 4-byte store); a block is four
// lanes, its maximum two shuffles.  A half warp has UNROLL such pieces in flight.  Scale bytes go to their places in the tiles one
// by one; L2 puts the words of neighbouring rows together.
// 2 or 4 bytes read and 17/32 written a value: bound by HBM.
#include "fp4.cuh"

namespace vptq {

namespace {

constexpr int THREADS = 256;

struct QuantizeParams {
    const void *x;
    int rows, cols;
    long long ld, pitch;
    int col_tiles;
    uint8_t *q, *scale;
    int early;
    long long step;            // pieces that all half warps take at a time, and the same as rows and tiles of columns
    int step_rows, step_cols;
};

template <int DT, bool VEC, int UNROLL>
__global__ void __launch_bounds__(THREADS)
fp4_quantize_kernel(const __grid_constant__ QuantizeParams P)
{
    if (P.early) pdl_launch_dependents();
    pdl_wait();
    // pieces of the matrix, rows after one another, are dealt out over the half warps; row and tile are counted on without divisions
    const int lane = threadIdx.x & 15, half = (threadIdx.x >> 4) & 1;
    const long long first = ((long long)blockIdx.x * THREADS + threadIdx.x) >> 4;
    int row = (int)(first / P.col_tiles), ct = (int)(first % P.col_tiles);
    const int last_tile = (P.rows - 1) / FP4_TILE_ROWS, last_rows = P.rows - last_tile * FP4_TILE_ROWS;
    // (a warp's two halves run the same number of rounds: shuffles)
    const long long n = (long long)P.rows * P.col_tiles;
    for (long long p0 = first - half; p0 < n; p0 += P.step * UNROLL) {
        Eight<DT, VEC> e[UNROLL];
        int rows[UNROLL], tiles[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; u++) {
            rows[u] = row; tiles[u] = ct;
            e[u] = load_eight<DT, VEC>(reinterpret_cast<const uint8_t *>(P.x) + (row < P.rows ? row : 0) * P.ld * Act<DT>::BYTES,
                                       row < P.rows ? ct * FP4_TILE_COLS + lane * 8 : P.cols, P.cols);
            ct += P.step_cols; row += P.step_rows;
            if (ct >= P.col_tiles) { ct -= P.col_tiles; row++; }
        }
#pragma unroll
        for (int u = 0; u < UNROLL; u++) {
            const uint32_t b = fp4_block_scale(magnitude(e[u]));
            if (rows[u] >= P.rows) continue;
            const int c = tiles[u] * FP4_TILE_COLS + lane * 8;
            float v[8];
            values_of(e[u], v);
            if (c / 2 < P.pitch) *reinterpret_cast<uint32_t *>(P.q + rows[u] * P.pitch + c / 2) = fp4_codes(v, b, P.cols - c);
            const int rt = rows[u] / FP4_TILE_ROWS, r = rows[u] % FP4_TILE_ROWS;
            uint8_t *tile = P.scale + ((long long)rt * P.col_tiles + tiles[u]) * FP4_TILE_BYTES;
            if ((lane & 3) == 0) tile[fp4_scale_at(r, lane >> 2)] = (uint8_t)b;
            // the last tile's rows that the matrix does not have: those a multiple of its rows behind this one are this half warp's
            if (rt == last_tile)
                for (int z = r + last_rows * (1 + lane); z < FP4_TILE_ROWS; z += last_rows * 16) *reinterpret_cast<uint32_t *>(tile + fp4_scale_at(z, 0)) = 0u;
        }
    }
}

template <int DT, bool VEC, int UNROLL>
cudaError_t launch_pieces(QuantizeParams P, long long ctas, cudaStream_t st)
{
    P.step = ctas * (THREADS / 16);
    P.step_rows = (int)(P.step / P.col_tiles);
    P.step_cols = (int)(P.step % P.col_tiles);
    return launch_dependent("fp4_quantize", fp4_quantize_kernel<DT, VEC, UNROLL>, (int)ctas, THREADS, 0, st, P);
}

template <int DT, bool VEC>
cudaError_t launch(const QuantizeParams &P, cudaStream_t st)
{
    // small calls: a piece per half warp; large ones: four in flight, on eight CTAs an SM
    const long long n = (long long)P.rows * P.col_tiles, per_cta = THREADS / 16;
    const long long resident = (long long)device_sm_count() * 8;
    const long long ctas = (n + per_cta - 1) / per_cta;
    if (ctas <= resident) return launch_pieces<DT, VEC, 1>(P, ctas, st);
    return launch_pieces<DT, VEC, 4>(P, (ctas + 3) / 4 < resident ? (ctas + 3) / 4 : resident, st);
}

}  // namespace

cudaError_t launch_fp4_quantize(const void *x, int x_dtype, int rows, int cols, long long ld, uint8_t *q, uint8_t *scale, bool early, cudaStream_t st)
{
    QuantizeParams P;
    P.x = x; P.rows = rows; P.cols = cols; P.ld = ld; P.pitch = fp4_row_bytes(cols);
    P.col_tiles = ceil_div(cols, FP4_TILE_COLS);
    P.q = q; P.scale = scale; P.early = early ? 1 : 0;
    const int bytes = x_dtype == VPTQ_DTYPE_FP32 ? 4 : 2, per = 16 / bytes;
    const bool vec = (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && cols % per == 0 && (rows == 1 || ld % per == 0);
    switch (x_dtype) {
    case VPTQ_DTYPE_FP16: return vec ? launch<VPTQ_DTYPE_FP16, true>(P, st) : launch<VPTQ_DTYPE_FP16, false>(P, st);
    case VPTQ_DTYPE_BF16: return vec ? launch<VPTQ_DTYPE_BF16, true>(P, st) : launch<VPTQ_DTYPE_BF16, false>(P, st);
    default: return vec ? launch<VPTQ_DTYPE_FP32, true>(P, st) : launch<VPTQ_DTYPE_FP32, false>(P, st);
    }
}

}  // namespace vptq
