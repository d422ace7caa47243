// Matrices in 8-bit floating point (e4m3) with a scale per block of 128 columns: the rule of the quantization and the pieces that
// the kernels over them share.
#pragma once
#include "common.cuh"

namespace vptq {

constexpr int FP8_BLOCK = 128;                            // columns (and rows, for weights) that share a scale
constexpr int FP8_MAX_SIZE = 1 << 30;                     // rows, columns, tokens: sums of a few of them stay in an int
constexpr float FP8_MAX = 448.f;                          // largest e4m3 value
constexpr float FP8_AMAX_MIN = 7.888609052210118e-31f;    // 2^-100: a block's largest value counts as at least this

inline long long fp8_row_bytes(long long cols) { return (cols + 15) / 16 * 16; }

// activations (or results) of `rows` rows to e4m3 with a scale per 128 columns of a row (block_rows = 1) or per 128 x 128 values
// (block_rows = 128); ld = distance of x's rows in values.  `early`: the kernel behind this one on the stream waits for it by itself
// before it touches q or scale.
cudaError_t launch_fp8_quantize(const void *x, int x_dtype, int rows, int cols, long long ld, int block_rows, uint8_t *q, float *scale,
                                bool early, cudaStream_t st);

// a vector-quantized layer to e4m3 with 128 x 128 blocks; inverse: null or N words of scratch (a stored column order needs them)
cudaError_t launch_dequant_fp8(const LayerView &L, uint8_t *q, float *scale, int *inverse, cudaStream_t st);

struct Fp8Linear {
    int M, N, B;
    int x_dtype, out_dtype;
    const void *x;
    const float *x_scale;      // e4m3 activations only
    const uint8_t *w;          // [M][fp8_row_bytes(N)]
    const float *w_scale;      // [ceil(M / 128)][ceil(N / 128)]
    void *out;
};

// Tokens of the decode kernel, one MMA's.  With 16 it took 52.6 us for 28672 x 8192 and 10.3 for 4096 x 4096, the tensor-core kernel behind
// a quantizing one 50.3 and 10.2 to 11.5.
constexpr int FP8_DECODE_MAX_B = 8;
cudaError_t launch_linear_fp8_decode(const Fp8Linear &P, cudaStream_t st);

long long linear_fp8_workspace_bytes(int N, int B, int x_dtype);
int linear_fp8_launches(int B, int x_dtype);
const char *linear_fp8_path(int B);
cudaError_t launch_linear_fp8(const Fp8Linear &P, void *ws, cudaStream_t st);

#ifdef __CUDACC__
// scale of a block whose largest magnitude is amax, and the factor its values are multiplied by before they are rounded to e4m3
struct Fp8Scale { float scale, factor; };
__device__ __forceinline__ Fp8Scale fp8_scale(float amax)
{
    const float a = amax < FP8_AMAX_MIN ? FP8_AMAX_MIN : amax;          // (a NaN stays)
    return {__fdiv_rn(a, FP8_MAX), __fdiv_rn(FP8_MAX, a)};
}

// Two values to e4m3, nearest, ties to even; beyond 448: 448; NaN: NaN.  lo in the low byte.
__device__ __forceinline__ uint32_t fp8_pair(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t fp8_quad(float a, float b, float c, float d) { return fp8_pair(a, b) | fp8_pair(c, d) << 16; }

// Types of activations.  `magnitude` keeps the largest magnitude of packed values as bits, in an order in which NaN > infinity >
// every number, so that one NaN or infinity shows in the block's scale.
template <int DT> struct Act;
template <> struct Act<VPTQ_DTYPE_FP16> {
    static constexpr int BYTES = 2;
    static __device__ __forceinline__ float2 two(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
    static __device__ __forceinline__ float one(const void *p, long long i) { return __half2float(reinterpret_cast<const __half *>(p)[i]); }
};
template <> struct Act<VPTQ_DTYPE_BF16> {
    static constexpr int BYTES = 2;
    static __device__ __forceinline__ float2 two(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
    static __device__ __forceinline__ float one(const void *p, long long i)
    {
        return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(p)[i] << 16);
    }
};
template <> struct Act<VPTQ_DTYPE_FP32> {
    static constexpr int BYTES = 4;
    static __device__ __forceinline__ float one(const void *p, long long i) { return reinterpret_cast<const float *>(p)[i]; }
};

// Eight consecutive values of a row, as they lie in memory (16-byte loads: VEC) or one by one as FP32.
template <int DT, bool VEC> struct Eight { float v[8]; };
template <> struct Eight<VPTQ_DTYPE_FP16, true> { uint4 q; };
template <> struct Eight<VPTQ_DTYPE_BF16, true> { uint4 q; };

// ... the first at column c of `cols`, zeros beyond; VEC: c and the row are aligned for it and cols is a multiple of a load's values
template <int DT, bool VEC>
__device__ __forceinline__ Eight<DT, VEC> load_eight(const void *row, int c, int cols)
{
    Eight<DT, VEC> e;
    if constexpr (VEC && DT == VPTQ_DTYPE_FP32) {
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const float4 q = c + i < cols ? __ldg(reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(row) + c + i)) : make_float4(0.f, 0.f, 0.f, 0.f);
            e.v[i] = q.x; e.v[i + 1] = q.y; e.v[i + 2] = q.z; e.v[i + 3] = q.w;
        }
    } else if constexpr (VEC) {
        e.q = c < cols ? __ldg(reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(row) + c)) : make_uint4(0, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) e.v[i] = c + i < cols ? Act<DT>::one(row, c + i) : 0.f;
    }
    return e;
}
template <int DT, bool VEC>
__device__ __forceinline__ void values_of(const Eight<DT, VEC> &e, float (&v)[8])
{
    if constexpr (VEC && DT != VPTQ_DTYPE_FP32) {
        const uint32_t w[4] = {e.q.x, e.q.y, e.q.z, e.q.w};
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const float2 f = Act<DT>::two(w[j]);
            v[2 * j] = f.x; v[2 * j + 1] = f.y;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = e.v[j];
    }
}

// larger magnitudes of two words of packed 16-bit values, low and high halves apart
__device__ __forceinline__ uint32_t max16(uint32_t a, uint32_t b) { return __vmaxu2(a & 0x7FFF7FFFu, b & 0x7FFF7FFFu); }
// ... and such a word's larger half as bits of an FP32 value
template <int DT>
__device__ __forceinline__ uint32_t magnitude16(uint32_t w)
{
    const uint32_t m = max(w & 0x7FFFu, (w >> 16) & 0x7FFFu);
    return DT == VPTQ_DTYPE_BF16 ? m << 16 : __float_as_uint(__half2float(__ushort_as_half((unsigned short)m)));
}

// largest magnitude of N values as bits
template <int N>
__device__ __forceinline__ uint32_t magnitude(const float (&v)[N])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; i++) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return m;
}
template <int DT, bool VEC>
__device__ __forceinline__ uint32_t magnitude(const Eight<DT, VEC> &e)
{
    if constexpr (VEC && DT != VPTQ_DTYPE_FP32) return magnitude16<DT>(max16(max16(e.q.x, e.q.y), max16(e.q.z, e.q.w)));
    else return magnitude<8>(e.v);
}
// eight values at column c of a row of q; beyond `cols` zeros are written up to the row's end, whatever the factor
template <int DT, bool VEC>
__device__ __forceinline__ void store_eight(uint8_t *row, long long pitch, int c, int cols, const Eight<DT, VEC> &e, float factor)
{
    if (c >= pitch) return;
    float v[8];
    values_of(e, v);
    uint2 o;
    o.x = fp8_quad(v[0] * factor, v[1] * factor, v[2] * factor, v[3] * factor);
    o.y = fp8_quad(v[4] * factor, v[5] * factor, v[6] * factor, v[7] * factor);
    *reinterpret_cast<uint2 *>(row + c) = o;
    if (c + 8 > cols)
        for (int i = max(c, cols); i < c + 8; i++) row[i] = 0;         // (0 * factor is no zero when the factor is a NaN)
}
#endif

}  // namespace vptq
