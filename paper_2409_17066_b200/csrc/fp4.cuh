// Matrices in 4-bit floating point (e2m1) with a power of two as the scale of every 32 columns of a row: the rule of the quantization,
// the order of the scales, and the pieces that the kernels over them share.
#pragma once
#include "fp8.cuh"

namespace vptq {

constexpr int FP4_BLOCK = 32;                             // columns of a row that share a scale
constexpr int FP4_TILE_ROWS = 128, FP4_TILE_COLS = 128;   // a tile of scales: 128 rows x 4 blocks of columns, 512 bytes
constexpr int FP4_TILE_BYTES = 512;

inline long long fp4_row_bytes(long long cols) { return (cols + FP4_BLOCK - 1) / FP4_BLOCK * (FP4_BLOCK / 2); }
inline long long fp4_scale_bytes(int rows, int cols)
{
    return (long long)ceil_div(rows, FP4_TILE_ROWS) * ceil_div(cols, FP4_TILE_COLS) * FP4_TILE_BYTES;
}

// `rows` rows to e2m1 (fp4_quantize.cu); ld = distance of x's rows in values.  The kernel behind this one on the
// stream may begin (and waits by itself before it touches q or scale) when this one has ended, at once, or when all those before this one have ended, what
// they have written with them.
enum class Behind { LAST, AT_ONCE, THEN };
cudaError_t launch_fp4_quantize(const void *x, int x_dtype, int rows, int cols, long long ld, uint8_t *q, uint8_t *scale, Behind behind, cudaStream_t st);
// ... and back to values [rows][cols] (fp4_values.cu)
cudaError_t launch_fp4_values(const uint8_t *q, const uint8_t *scale, int rows, int cols, int out_dtype, void *out, cudaStream_t st);

// a vector-quantized layer to e2m1 (dequant_fp8.cu); inverse: null or N words of scratch (a stored column order needs them)
cudaError_t launch_dequant_fp4(const LayerView &L, uint8_t *q, uint8_t *scale, int *inverse, cudaStream_t st);
// ... of the layers whose columns lie as they are stored (dequant_fp4.cu)
bool dequant_fp4_takes(const LayerView &L);
cudaError_t launch_dequant_fp4_rows(const LayerView &L, uint8_t *q, uint8_t *scale, cudaStream_t st);

struct Fp4Linear {
    int M, N, B;
    int x_dtype, out_dtype;
    const void *x;
    const uint8_t *x_scale;    // e2m1 activations only
    const uint8_t *w, *w_scale;
    void *out;
};
long long linear_fp4_workspace_bytes(int M, int N, int B, int x_dtype);
int linear_fp4_launches(int M, int N, int B, int x_dtype);
const char *linear_fp4_path(int M, int N, int B, int x_dtype);
cudaError_t launch_linear_fp4(const Fp4Linear &P, void *ws, cudaStream_t st);

#ifdef __CUDACC__
// byte of row r (of 128) and block k (of 4) in its tile: the tensor cores take a lane's four rows 32 apart
__device__ __forceinline__ int fp4_scale_at(int r, int k) { return (r & 31) * 16 + (r >> 5) * 4 + k; }

// The scale byte b of a block whose largest magnitude has these FP32 bits; it stands for 2^(b - 127).  That magnitude is in [3.5, 7) times
// the scale: no value is cut at 6 by more than the half step that rounding may take, and the top code is in use whenever it can be.  Rounding the
// mantissa up from 1.75 is one addition.  An infinity or a NaN: 255, which stands for NaN.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t amax)
{
    if (amax >= 0x7F800000u) return 255u;
    const int b = (int)((amax + 0x00200000u) >> 23) - 2;
    return b > 0 ? (uint32_t)b : 0u;
}
// 1 / scale: a power of two in FP32's normal range for every b of a finite block (0 to 253)
__device__ __forceinline__ float fp4_factor(uint32_t b) { return __uint_as_float((254u - b) << 23); }
__device__ __forceinline__ float fp4_scale_value(uint32_t b)
{
    return __uint_as_float(b == 255u ? 0x7FFFFFFFu : b == 0u ? 0x00400000u : b << 23);
}

// (a * f, b * f), two products in one instruction
__device__ __forceinline__ void times2(float &x, float &y, float a, float b, float f)
{
    asm("{\n\t.reg .b64 v, s;\n\tmov.b64 v, {%2, %3};\n\tmov.b64 s, {%4, %4};\n\tmul.rn.f32x2 v, v, s;\n\tmov.b64 {%0, %1}, v;\n\t}" : "=f"(x), "=f"(y) : "f"(a), "f"(b), "f"(f));
}

// Eight values to codes, nearest, ties to even, at most 6; v[0] in the lowest four bits.
__device__ __forceinline__ uint32_t fp4_eight(const float (&v)[8])
{
    uint32_t r;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// ... and back; every code is exact in FP16
__device__ __forceinline__ void fp4_values8(uint32_t q, float (&v)[8])
{
    uint32_t h[4];
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\tcvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(q));
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[i]));
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
}

// Sixteen consecutive values of a row, as two times eight; zeros beyond `cols`.  Values of 16 bits are packed whether they were loaded so (VEC: 16 bytes at a
// time) or in words, or halves of them at the ends, that lie anywhere.
template <int DT, bool VEC> struct Sixteen { Eight<DT, VEC || DT != VPTQ_DTYPE_FP32> h[2]; };
template <int DT, bool VEC>
__device__ __forceinline__ Sixteen<DT, VEC> load_sixteen(const void *row, int c, int cols)
{
    if constexpr (VEC || DT == VPTQ_DTYPE_FP32) {
        return {{load_eight<DT, VEC>(row, c, cols), load_eight<DT, VEC>(row, c + 8, cols)}};
    } else {
        const uint16_t *p = reinterpret_cast<const uint16_t *>(row) + c;
        uint32_t w[8] = {};
        if (c + 16 <= cols) {
            if ((reinterpret_cast<uintptr_t>(p) & 2u) == 0) {
#pragma unroll
                for (int i = 0; i < 8; i++) w[i] = __ldg(reinterpret_cast<const uint32_t *>(p) + i);
            } else {
                // a half, seven words, a half: no value beside these is touched
                uint32_t last = __ldg(p);
#pragma unroll
                for (int i = 0; i < 7; i++) {
                    const uint32_t next = __ldg(reinterpret_cast<const uint32_t *>(p + 1) + i);
                    w[i] = i == 0 ? last | next << 16 : __funnelshift_r(last, next, 16);
                    last = next;
                }
                w[7] = last >> 16 | (uint32_t)__ldg(p + 15) << 16;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; i++)
                if (c + i < cols) w[i / 2] |= (uint32_t)__ldg(p + i) << (16 * (i & 1));
        }
        Sixteen<DT, VEC> e;
        e.h[0].q = make_uint4(w[0], w[1], w[2], w[3]);
        e.h[1].q = make_uint4(w[4], w[5], w[6], w[7]);
        return e;
    }
}
// the larger magnitudes of two words of packed 16-bit values, whose signs are cleared
__device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b)
{
    asm("max.u16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
    return a;
}
// their largest magnitude, as bits of an FP32 value in which NaN > infinity > every number
template <int DT, bool VEC>
__device__ __forceinline__ uint32_t magnitude(const Sixteen<DT, VEC> &e)
{
    if constexpr (DT != VPTQ_DTYPE_FP32) {
        const uint32_t w[8] = {e.h[0].q.x, e.h[0].q.y, e.h[0].q.z, e.h[0].q.w, e.h[1].q.x, e.h[1].q.y, e.h[1].q.z, e.h[1].q.w};
        uint32_t m = w[0] & 0x7FFF7FFFu;
#pragma unroll
        for (int i = 1; i < 8; i++) m = larger2(m, w[i] & 0x7FFF7FFFu);
        return magnitude16<DT>(m);
    } else {
        return max(magnitude<8>(e.h[0].v), magnitude<8>(e.h[1].v));        // (an Eight of FP32 is the values)
    }
}
// Two lanes, OTHER apart, hold a block's 32 values: its scale byte.
template <int OTHER = 1>
__device__ __forceinline__ uint32_t fp4_pair_scale(uint32_t m) { return fp4_scale_byte(max(m, __shfl_xor_sync(0xffffffffu, m, OTHER))); }

// Four adjacent lanes hold a block's 32 values: its scale byte, from each lane's largest magnitude (as bits).
__device__ __forceinline__ uint32_t fp4_block_scale(uint32_t m)
{
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    return fp4_scale_byte(m);
}
// Codes of eight values of a block with scale byte b, of which the first `n` exist (the others are zeros).  A block that is not finite
// holds the top code throughout, which reads as NaN.
__device__ __forceinline__ uint32_t fp4_codes(const float (&v)[8], uint32_t b, int n)
{
    if (b == 255u) return n >= 8 ? 0x77777777u : n <= 0 ? 0u : 0x77777777u & ((1u << (4 * n)) - 1u);
    const float f = fp4_factor(b);
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) times2(t[i], t[i + 1], v[i], v[i + 1], f);
    return fp4_eight(t);
}

// codes of sixteen values, of which the first `n` exist
template <int DT, bool VEC>
__device__ __forceinline__ uint2 fp4_codes16(const Sixteen<DT, VEC> &e, uint32_t b, int n)
{
    float lo[8], hi[8];
    values_of(e.h[0], lo);
    values_of(e.h[1], hi);
    return make_uint2(fp4_codes(lo, b, n), fp4_codes(hi, b, n - 8));
}

// values of eight codes times their scale
__device__ __forceinline__ void fp4_scaled8(uint32_t q, float s, float (&v)[8])
{
    fp4_values8(q, v);
#pragma unroll
    for (int i = 0; i < 8; i += 2) times2(v[i], v[i + 1], v[i], v[i + 1], s);
}

// eight FP32 values as four words of 16-bit ones
template <int DT>
__device__ __forceinline__ void pack16(const float (&v)[8], uint32_t (&w)[4])
{
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if constexpr (DT == VPTQ_DTYPE_FP16) {
            const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&h);
        } else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
    }
}
// 32 bytes on a boundary of 32
__device__ __forceinline__ void store32(void *p, const uint32_t (&a)[4], const uint32_t (&b)[4])
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]), "r"(b[2]), "r"(b[3]) : "memory");
}

// eight values to `out` at column c of a row of `cols` values; VEC: the row starts on 16 bytes and cols is a multiple of a store's values
template <int DT, bool VEC>
__device__ __forceinline__ void store_values8(void *row, int c, int cols, const float (&v)[8])
{
    if (c >= cols) return;
    if constexpr (VEC && DT == VPTQ_DTYPE_FP32) {
        float4 *p = reinterpret_cast<float4 *>(reinterpret_cast<float *>(row) + c);
        __stcs(p, make_float4(v[0], v[1], v[2], v[3]));
        if (c + 4 < cols) __stcs(p + 1, make_float4(v[4], v[5], v[6], v[7]));
    } else if constexpr (VEC) {
        uint32_t w[4];
        pack16<DT>(v, w);
        __stcs(reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(row) + c), make_uint4(w[0], w[1], w[2], w[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (c + i < cols) store_out(row, c + i, v[i], DT);
    }
}
// Sixteen values to `out` at column c of a row of `cols` values.  wide: the row starts on 32 bytes and cols is a multiple of 16.
template <int DT, bool VEC>
__device__ __forceinline__ void store_values16(void *row, int c, int cols, bool wide, const float (&lo)[8], const float (&hi)[8])
{
    if (VEC && wide) {
        if constexpr (DT == VPTQ_DTYPE_FP32) {
#pragma unroll
            for (int i = 0; i < 2; i++) {
                uint32_t a[4], b[4];
#pragma unroll
                for (int k = 0; k < 4; k++) { a[k] = __float_as_uint(i ? hi[k] : lo[k]); b[k] = __float_as_uint(i ? hi[4 + k] : lo[4 + k]); }
                store32(reinterpret_cast<float *>(row) + c + 8 * i, a, b);
            }
        } else {
            uint32_t a[4], b[4];
            pack16<DT>(lo, a);
            pack16<DT>(hi, b);
            store32(reinterpret_cast<uint16_t *>(row) + c, a, b);
        }
    } else {
        store_values8<DT, VEC>(row, c, cols, lo);
        store_values8<DT, VEC>(row, c + 8, cols, hi);
    }
}
#endif

}  // namespace vptq
