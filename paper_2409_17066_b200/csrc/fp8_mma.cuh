// Products of an e4m3 weight with a few e4m3 activations in one warp (mma.sync m16n8k32): the core of the decode kernel and of the
// mixture-of-experts kernels.
//
// A warp takes 16 weight rows and 8 tokens, 128 columns (one scale block) at a time.  The order of the products inside a block is
// free, so a lane's operands are 16-byte pieces as they lie in memory: lane 4g + t holds bytes 16t .. 16t+15 of each 64-byte half of
// rows g and g + 8 and of token g's values, and MMA 2c + h of the block takes words 2h and 2h + 1 of half c.
#pragma once
#include "fp8.cuh"

namespace vptq {

#ifdef __CUDACC__
__device__ __forceinline__ uint4 load_stream16(const uint8_t *p)
{
    uint4 q;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(p));
    return q;
}

__device__ __forceinline__ void mma_e4m3(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A lane's share of 16 weight rows in one block: [row g or g + 8][half]
struct WeightFrag { uint4 q[2][2]; };
// `at` = offset of the lane's piece of the block's first half in a row; rows of `pitch` bytes, whose pad bytes are zeros
__device__ __forceinline__ WeightFrag load_weights(const uint8_t *row_g, const uint8_t *row_g8, long long at, long long pitch)
{
    WeightFrag f;
#pragma unroll
    for (int c = 0; c < 2; c++) {
        const bool in = at + 64 * c < pitch;
        f.q[0][c] = in ? load_stream16(row_g + at + 64 * c) : make_uint4(0, 0, 0, 0);
        f.q[1][c] = in ? load_stream16(row_g8 + at + 64 * c) : make_uint4(0, 0, 0, 0);
    }
    return f;
}

// A lane's share of one token's values in one block, as they lie in memory
template <int DT, bool VEC> struct TokenRaw { float v[32]; };                         // (value by value)
template <> struct TokenRaw<VPTQ_DTYPE_FP16, true> { uint4 q[4]; };
template <> struct TokenRaw<VPTQ_DTYPE_BF16, true> { uint4 q[4]; };
template <> struct TokenRaw<VPTQ_DTYPE_FP32, true> { float4 q[8]; };
template <bool VEC> struct TokenRaw<VPTQ_DTYPE_E4M3, VEC> { uint4 q[2]; float scale; };

// ... and as MMA operands with the block's scale
struct TokenFrag { uint32_t w[8]; float scale; };

// row: the token's values, or null for a token that is not there (zeros); kb: block, t: lane & 3; cols: values of a row (e4m3: its pitch)
template <int DT, bool VEC>
__device__ __forceinline__ TokenRaw<DT, VEC> load_token(const void *row, const float *scales, int kb, int t, int cols)
{
    TokenRaw<DT, VEC> r;
    const int c0 = kb * FP8_BLOCK + 16 * t;
    if constexpr (DT == VPTQ_DTYPE_E4M3) {
        r.scale = row != nullptr ? __ldg(scales + kb) : 0.f;
#pragma unroll
        for (int c = 0; c < 2; c++)
            r.q[c] = row != nullptr && c0 + 64 * c < cols ? __ldg(reinterpret_cast<const uint4 *>(reinterpret_cast<const uint8_t *>(row) + c0 + 64 * c)) : make_uint4(0, 0, 0, 0);
    } else if constexpr (!VEC) {
#pragma unroll
        for (int i = 0; i < 32; i++) {
            const int c = c0 + 64 * (i >> 4) + (i & 15);
            r.v[i] = row != nullptr && c < cols ? Act<DT>::one(row, c) : 0.f;
        }
    } else if constexpr (DT == VPTQ_DTYPE_FP32) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int c = c0 + 64 * (i >> 2) + 4 * (i & 3);
            r.q[i] = row != nullptr && c < cols ? __ldcg(reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(row) + c)) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int c = c0 + 64 * (i >> 1) + 8 * (i & 1);
            r.q[i] = row != nullptr && c < cols ? __ldg(reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(row) + c)) : make_uint4(0, 0, 0, 0);
        }
    }
    return r;
}

// The four lanes of a token share the block's 128 values: its maximum is two shuffles away (every lane of the warp calls this).
template <int DT, bool VEC>
__device__ __forceinline__ TokenFrag quantize_token(const TokenRaw<DT, VEC> &r)
{
    TokenFrag f;
    if constexpr (DT == VPTQ_DTYPE_E4M3) {
        f.scale = r.scale;
#pragma unroll
        for (int c = 0; c < 2; c++) { f.w[4 * c] = r.q[c].x; f.w[4 * c + 1] = r.q[c].y; f.w[4 * c + 2] = r.q[c].z; f.w[4 * c + 3] = r.q[c].w; }
    } else {
        float v[32];
        if constexpr (!VEC) {
#pragma unroll
            for (int i = 0; i < 32; i++) v[i] = r.v[i];
        } else if constexpr (DT == VPTQ_DTYPE_FP32) {
#pragma unroll
            for (int i = 0; i < 8; i++) { v[4 * i] = r.q[i].x; v[4 * i + 1] = r.q[i].y; v[4 * i + 2] = r.q[i].z; v[4 * i + 3] = r.q[i].w; }
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t w[4] = {r.q[i].x, r.q[i].y, r.q[i].z, r.q[i].w};
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const float2 p = Act<DT>::two(w[j]);
                    v[8 * i + 2 * j] = p.x; v[8 * i + 2 * j + 1] = p.y;
                }
            }
        }
        uint32_t m = magnitude<32>(v);
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
        const Fp8Scale s = fp8_scale(__uint_as_float(m));
        f.scale = s.scale;
#pragma unroll
        for (int i = 0; i < 8; i++) f.w[i] = fp8_quad(v[4 * i] * s.factor, v[4 * i + 1] * s.factor, v[4 * i + 2] * s.factor, v[4 * i + 3] * s.factor);
    }
    return f;
}

// acc += (the block's products of 16 rows and 8 tokens) * weight scale * token scale.  acc: rows g, g + 8 of tokens 2t, 2t + 1 as
// [g][2t], [g][2t+1], [g+8][2t], [g+8][2t+1]; s0, s1 = the two tokens' scales times the weight's.
__device__ __forceinline__ void block_product(float (&acc)[4], const WeightFrag &a, const TokenFrag &b, float s0, float s1)
{
    float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 2; c++) {
        mma_e4m3(d, a.q[0][c].x, a.q[1][c].x, a.q[0][c].y, a.q[1][c].y, b.w[4 * c], b.w[4 * c + 1]);
        mma_e4m3(d, a.q[0][c].z, a.q[1][c].z, a.q[0][c].w, a.q[1][c].w, b.w[4 * c + 2], b.w[4 * c + 3]);
    }
    acc[0] = __fmaf_rn(d[0], s0, acc[0]); acc[1] = __fmaf_rn(d[1], s1, acc[1]);
    acc[2] = __fmaf_rn(d[2], s0, acc[2]); acc[3] = __fmaf_rn(d[3], s1, acc[3]);
}
// the scales of the tokens that a lane's accumulators belong to (token i's scale is known to lanes 4i .. 4i+3)
__device__ __forceinline__ float2 scales_of_columns(float scale, int t)
{
    return make_float2(__shfl_sync(0xffffffffu, scale, 8 * t), __shfl_sync(0xffffffffu, scale, 8 * t + 4));
}
#endif

}  // namespace vptq
