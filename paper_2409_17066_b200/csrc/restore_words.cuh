// What the kernels that restore weights (dequant.cu, dequant_fp8.cu) share: a lane's indices as a window of packed words, table rows as
// words, the residual's addition.
#pragma once
#include "common.cuh"

namespace vptq {

// One table row of V values as words; `e` counts rows of 2V bytes in global memory.
template <int V> struct RowWords { uint32_t w[V > 0 ? (V + 1) / 2 : 1]; };

template <int V>
__device__ __forceinline__ RowWords<V> row_from_global(const __half *__restrict__ tab, long long e)
{
    RowWords<V> r;
    if (V == 8) {
        const uint4 q = __ldg(reinterpret_cast<const uint4 *>(tab) + e);
        r.w[0] = q.x; r.w[1] = q.y; r.w[2] = q.z; r.w[V / 2 - 1] = q.w;
    } else if (V % 4 == 0) {
        const uint2 *p = reinterpret_cast<const uint2 *>(tab) + e * (V / 4);
#pragma unroll
        for (int i = 0; i < V / 4; i++) { const uint2 q = __ldg(p + i); r.w[2 * i] = q.x; r.w[2 * i + 1] = q.y; }
    } else {
        const uint32_t *p = reinterpret_cast<const uint32_t *>(tab) + e * (V / 2);
#pragma unroll
        for (int i = 0; i < V / 2; i++) r.w[i] = __ldg(p + i);
    }
    return r;
}

// The packed bits of CPL consecutive indices, the first at stream bit `bit`: words beyond the row read as zero.
template <int CPL>
struct IndexWindow { uint32_t w[CPL / 2 + 1]; };
template <int CPL>
__device__ __forceinline__ IndexWindow<CPL> load_window(const uint8_t *__restrict__ row, unsigned bit, unsigned row_words)
{
    IndexWindow<CPL> q;
    const unsigned w0 = bit >> 5;
#pragma unroll
    for (int i = 0; i <= CPL / 2; i++) q.w[i] = w0 + i < row_words ? __ldg(reinterpret_cast<const uint32_t *>(row) + w0 + i) : 0u;
    return q;
}
// ... and index s of it, for widths of 8, 12 and 16 bits (`sh` = bit & 31), clamped to k - 1
template <int CPL>
__device__ __forceinline__ void decode_window(const IndexWindow<CPL> &q, unsigned sh, int bits, int k, int (&idx)[CPL])
{
    const uint32_t lim = (uint32_t)(k - 1);
    uint32_t a[CPL / 2 + 1];
#pragma unroll
    for (int i = 0; i < CPL / 2; i++) a[i] = __funnelshift_r(q.w[i], q.w[i + 1], sh);
    a[CPL / 2] = 0;
    if (bits == 16) {
#pragma unroll
        for (int s = 0; s < CPL; s++) idx[s] = (int)min((s & 1) ? a[s >> 1] >> 16 : a[s >> 1] & 0xFFFFu, lim);
    } else if (bits == 12) {
#pragma unroll
        for (int s = 0; s < CPL; s++)
            idx[s] = (int)min(__funnelshift_r(a[(12 * s) >> 5], a[((12 * s) >> 5) + 1], (12 * s) & 31) & 0xFFFu, lim);
    } else {
#pragma unroll
        for (int s = 0; s < CPL; s++) idx[s] = (int)min((a[s >> 2] >> (8 * (s & 3))) & 0xFFu, lim);
    }
}

// c + (the two halves of w), rounded once: w * 1 is exact
__device__ __forceinline__ float2 add_half2(float2 c, uint32_t w)
{
    asm("{\n\t.reg .b16 lo, hi, one;\n\tmov.b32 {lo, hi}, %2;\n\tmov.b16 one, 0x3C00;\n\t"
        "fma.rn.f32.f16 %0, lo, one, %0;\n\tfma.rn.f32.f16 %1, hi, one, %1;\n\t}" : "+f"(c.x), "+f"(c.y) : "r"(w));
    return c;
}

}  // namespace vptq
