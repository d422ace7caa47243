// Quantization to e2m1 with a power of two for every 32 columns of a row: the block's largest magnitude gives the scale by one integer
// addition (fp4.cuh), the codes are the hardware's conversion of x / scale, which is exact before it is rounded.
//
// A CTA makes one tile of scales, 128 rows x 128 columns: a lane takes sixteen adjacent columns (two 16-byte loads of 16-bit values, an 8-byte
// store), two lanes are a block, eight a row, and a thread has four rows, 32 apart as the tile wants them, all four in flight.  Rows that the
// matrix does not have are zeros and give the zeros that the tile holds there.
// 2 or 4 bytes read and 17/32 written a value: bound by HBM, once the instructions are few.  (Eight columns to a lane and four lanes to a block, which
// is one more shuffle and twice the address arithmetic a value, took 146 us instead of 88, 6.8 TB/s, for 28672 x 8192 from 16 bits.)
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
    Behind behind;
};

// STEPS: rows of a thread; a tile is 4 / STEPS CTAs' work
template <int DT, bool VEC, int STEPS>
__global__ void __launch_bounds__(THREADS)
fp4_quantize_kernel(const __grid_constant__ QuantizeParams P)
{
    if (P.behind == Behind::AT_ONCE) pdl_launch_dependents();
    pdl_wait();
    if (P.behind == Behind::THEN) pdl_launch_dependents();
    const int lane = threadIdx.x & 7, r = threadIdx.x >> 3;
    const unsigned tile = STEPS == 4 ? blockIdx.x : blockIdx.x / (4 / STEPS);
    const int rt = (int)(tile / (unsigned)P.col_tiles), ct = (int)(tile - (unsigned)rt * P.col_tiles), j0 = STEPS == 4 ? 0 : (int)(blockIdx.x % (4 / STEPS)) * STEPS;
    const int row = rt * FP4_TILE_ROWS + 32 * j0 + r, c = ct * FP4_TILE_COLS + lane * 16;
    const uint8_t *x = reinterpret_cast<const uint8_t *>(P.x) + (long long)row * P.ld * Act<DT>::BYTES;
    uint8_t *q = P.q + (long long)row * P.pitch + c / 2, *scale = P.scale + (long long)tile * FP4_TILE_BYTES + fp4_scale_at(32 * j0 + r, lane >> 1);
    const long long step = 32 * P.ld * Act<DT>::BYTES;
    Sixteen<DT, VEC> e[STEPS];
#pragma unroll
    for (int j = 0; j < STEPS; j++) e[j] = load_sixteen<DT, VEC>(x + j * step, row + 32 * j < P.rows ? c : P.cols, P.cols);
#pragma unroll
    for (int j = 0; j < STEPS; j++) {
        const uint32_t b = fp4_pair_scale(magnitude(e[j]));
        if (row + 32 * j < P.rows && c / 2 < P.pitch) *reinterpret_cast<uint2 *>(q + j * 32 * P.pitch) = fp4_codes16(e[j], b, P.cols - c);
        if ((lane & 1) == 0) scale[4 * j] = (uint8_t)b;
    }
}

// Where whole tiles would not give every SM two CTAs, a row to a thread (500 x 4096 in 512 CTAs 1.8 us).
template <int DT, bool VEC>
cudaError_t launch_as(const QuantizeParams &P, cudaStream_t st)
{
    const int tiles = (int)((long long)ceil_div(P.rows, FP4_TILE_ROWS) * P.col_tiles);
    if (tiles < 2 * device_sm_count()) return launch_dependent("fp4_quantize", fp4_quantize_kernel<DT, VEC, 1>, 4 * tiles, THREADS, 0, st, P);
    return launch_dependent("fp4_quantize", fp4_quantize_kernel<DT, VEC, 4>, tiles, THREADS, 0, st, P);
}
template <int DT>
cudaError_t launch(const QuantizeParams &P, bool vec, cudaStream_t st) { return vec ? launch_as<DT, true>(P, st) : launch_as<DT, false>(P, st); }

}  // namespace

cudaError_t launch_fp4_quantize(const void *x, int x_dtype, int rows, int cols, long long ld, uint8_t *q, uint8_t *scale, Behind behind, cudaStream_t st)
{
    QuantizeParams P;
    P.x = x; P.rows = rows; P.cols = cols; P.ld = ld; P.pitch = fp4_row_bytes(cols);
    P.col_tiles = ceil_div(cols, FP4_TILE_COLS);
    P.q = q; P.scale = scale; P.behind = behind;
    const int bytes = x_dtype == VPTQ_DTYPE_FP32 ? 4 : 2, per = 16 / bytes;
    const bool vec = (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && cols % per == 0 && (rows == 1 || ld % per == 0);
    switch (x_dtype) {
    case VPTQ_DTYPE_FP16: return launch<VPTQ_DTYPE_FP16>(P, vec, st);
    case VPTQ_DTYPE_BF16: return launch<VPTQ_DTYPE_BF16>(P, vec, st);
    default: return launch<VPTQ_DTYPE_FP32>(P, vec, st);
    }
}

}  // namespace vptq
