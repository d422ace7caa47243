// Values of an e2m1 matrix: code times its block's power of two, exact in FP32, rounded once to the result's type.
//
// A lane takes eight adjacent columns: four bytes of codes, one scale byte, a 16-byte store of 16-bit values; UNROLL rows of a tile at
// a time, so that as many reads are in flight.  17/32 of a byte read and 2 or 4 written a value: bound by HBM's writes (28672 x 8192 to 16 bits 89 us,
// 6.7 TB/s).
// Rows that are no multiples of 16 bytes: the result is one run of values, of which a lane takes eight on a boundary of 16 bytes wherever in a row they begin; their
// codes are a window of two words, of two blocks at most.  (Row by row with a store a value: 4096 x 4095
// 53 us, 18 so.)
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

template <int DT>
__device__ __forceinline__ void store_run(void *out, long long at, const float (&v)[8])
{
    if constexpr (DT == VPTQ_DTYPE_FP32) {
        float4 *p = reinterpret_cast<float4 *>(reinterpret_cast<float *>(out) + at);
        __stcs(p, make_float4(v[0], v[1], v[2], v[3]));
        __stcs(p + 1, make_float4(v[4], v[5], v[6], v[7]));
    } else {
        uint32_t w[4];
        pack16<DT>(v, w);
        __stcs(reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(out) + at), make_uint4(w[0], w[1], w[2], w[3]));
    }
}

template <int DT>
__global__ void __launch_bounds__(THREADS)
fp4_values_run_kernel(const __grid_constant__ ValuesParams P)
{
    pdl_wait();
    const long long total = (long long)P.rows * P.cols;
    const long long at = ((long long)blockIdx.x * THREADS + threadIdx.x) * 8;
    if (at >= total) return;
    const long long row = total < 1ll << 32 ? (uint32_t)at / (uint32_t)P.cols : at / P.cols;
    const int c = (int)(at - row * P.cols);
    auto scale_byte = [&](long long row, int c) {
        return __ldg(P.scale + (row / FP4_TILE_ROWS * P.col_tiles + c / FP4_TILE_COLS) * FP4_TILE_BYTES + fp4_scale_at((int)(row % FP4_TILE_ROWS), c / FP4_BLOCK % 4));
    };
    if (c + 8 <= P.cols) {
        // (a second word or block is only asked for where the row has columns of it)
        const uint32_t *q = reinterpret_cast<const uint32_t *>(P.q + row * P.pitch) + c / 8;
        const int inside = c % 8, first = min(8, FP4_BLOCK - c % FP4_BLOCK);
        const uint32_t w0 = __ldg(q), w1 = inside ? __ldg(q + 1) : 0u;
        const float s0 = fp4_scale_value(scale_byte(row, c)), s1 = first < 8 ? fp4_scale_value(scale_byte(row, c + first)) : s0;
        float v[8];
        fp4_values8(__funnelshift_r(w0, w1, 4 * inside), v);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] *= i < first ? s0 : s1;
        store_run<DT>(P.out, at, v);
    } else {
        uint32_t code[8], byte[8];
        int k = c;
        long long r = row;
#pragma unroll
        for (int i = 0; i < 8; i++, k++) {
            if (k == P.cols) { k = 0; r++; }
            const bool in = at + i < total;
            code[i] = in ? __ldg(P.q + r * P.pitch + k / 2) >> (4 * (k & 1)) & 15u : 0u;
            byte[i] = in ? scale_byte(r, k) : 0u;
        }
        uint32_t q = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) q |= code[i] << (4 * i);
        float v[8];
        fp4_values8(q, v);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] *= fp4_scale_value(byte[i]);
        if (at + 8 <= total) store_run<DT>(P.out, at, v);
        else
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (at + i < total) store_out(P.out, at + i, v[i], DT);
    }
}

template <int DT>
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
        store_values8<DT, true>(reinterpret_cast<uint8_t *>(P.out) + (long long)row * P.cols * (DT == VPTQ_DTYPE_FP32 ? 4 : 2), c, P.cols, v);
    }
}

template <int DT>
cudaError_t launch(const ValuesParams &P, cudaStream_t st)
{
    const long long ctas = (long long)ceil_div(P.rows, ROWS) * P.col_tiles;
    if (P.cols % (DT == VPTQ_DTYPE_FP32 ? 4 : 8) == 0) return launch_dependent("fp4_values", fp4_values_kernel<DT>, (int)ctas, THREADS, 0, st, P);
    const long long run = 8ll * THREADS;
    return launch_dependent("fp4_values", fp4_values_run_kernel<DT>, (int)(((long long)P.rows * P.cols + run - 1) / run), THREADS, 0, st, P);
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
