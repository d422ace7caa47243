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
__device__ __forceinline__ void mma_e4m3(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A lane's share of 16 weight rows in one block: [row g or g + 8][half]
struct WeightFrag { uint4 q[2][2]; };
// A lane's share of one token's values in one block, as they lie in memory
template <int DT, bool VEC> struct TokenRaw { float v[32]; };                         // (value by value)
template <> struct TokenRaw<VPTQ_DTYPE_FP16, true> { uint4 q[4]; };
template <> struct TokenRaw<VPTQ_DTYPE_BF16, true> { uint4 q[4]; };
template <bool VEC> struct TokenRaw<VPTQ_DTYPE_E4M3, VEC> { uint4 q[2]; };

// ... and as MMA operands with the block's scale
struct TokenFrag { uint32_t w[8]; float scale; };

// row: the token's values, or null for a token that is not there (zeros); kb: block, t: lane & 3; cols: values of a row (e4m3: its pitch)
template <int DT, bool VEC>
__device__ __forceinline__ TokenRaw<DT, VEC> load_token(const void *row, int t, int kb, int cols)
{
    TokenRaw<DT, VEC> r;
    const int c0 = kb * FP8_BLOCK + 16 * t;
    if constexpr (DT == VPTQ_DTYPE_E4M3) {
#pragma unroll
        for (int c = 0; c < 2; c++)
            r.q[c] = row != nullptr && c0 + 64 * c < cols ? __ldg(reinterpret_cast<const uint4 *>(reinterpret_cast<const uint8_t *>(row) + c0 + 64 * c)) : make_uint4(0, 0, 0, 0);
    } else if constexpr (!VEC) {
#pragma unroll
        for (int i = 0; i < 32; i++) {
            const int c = c0 + 64 * (i >> 4) + (i & 15);
            r.v[i] = row != nullptr && c < cols ? Act<DT>::one(row, c) : 0.f;
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
// scale: of a block that is in e4m3 already.
template <int DT, bool VEC>
__device__ __forceinline__ TokenFrag quantize_token(const TokenRaw<DT, VEC> &r, float scale)
{
    TokenFrag f;
    if constexpr (DT == VPTQ_DTYPE_E4M3) {
        f.scale = scale;
#pragma unroll
        for (int c = 0; c < 2; c++) { f.w[4 * c] = r.q[c].x; f.w[4 * c + 1] = r.q[c].y; f.w[4 * c + 2] = r.q[c].z; f.w[4 * c + 3] = r.q[c].w; }
    } else {
        float v[32];
        if constexpr (!VEC) {
#pragma unroll
            for (int i = 0; i < 32; i++) v[i] = r.v[i];
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
        uint32_t m;
        if constexpr (VEC) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = max16(max16(r.q[i].x, r.q[i].y), max16(r.q[i].z, r.q[i].w));
            m = magnitude16<DT>(max16(max16(w[0], w[1]), max16(w[2], w[3])));
        } else {
            m = magnitude<32>(v);
        }
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
        const Fp8Scale s = fp8_scale(__uint_as_float(m));
        f.scale = s.scale;
#pragma unroll
        for (int i = 0; i < 8; i++) f.w[i] = fp8_quad(v[4 * i] * s.factor, v[4 * i + 1] * s.factor, v[4 * i + 2] * s.factor, v[4 * i + 3] * s.factor);
    }
    return f;
}

// For each of R groups of 16 rows and N of 8 tokens: acc += (the block's products) * scale.  A lane's four sums of a pair are rows g,
// g + 8 of tokens 2t, 2t + 1 as [g][2t], [g][2t+1], [g+8][2t], [g+8][2t+1]; scale(r, n) gives the two tokens' scales times the weight's.
// Step by step over all pairs: the four MMAs of a pair wait for one another.
template <int R, int N, typename Scale>
__device__ __forceinline__ void block_products(float (*acc)[N][4], const WeightFrag (&a)[R], const TokenFrag (&b)[N], Scale scale)
{
    float d[R][N][4] = {};
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
        for (int r = 0; r < R; r++)
#pragma unroll
            for (int n = 0; n < N; n++) {
                const uint4 &p = a[r].q[0][i >> 1], &q = a[r].q[1][i >> 1];
                if (i & 1) mma_e4m3(d[r][n], p.z, q.z, p.w, q.w, b[n].w[2 * i], b[n].w[2 * i + 1]);
                else mma_e4m3(d[r][n], p.x, q.x, p.y, q.y, b[n].w[2 * i], b[n].w[2 * i + 1]);
            }
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
        for (int n = 0; n < N; n++) {
            const float2 s = scale(r, n);
            acc[r][n][0] = __fmaf_rn(d[r][n][0], s.x, acc[r][n][0]); acc[r][n][1] = __fmaf_rn(d[r][n][1], s.y, acc[r][n][1]);
            acc[r][n][2] = __fmaf_rn(d[r][n][2], s.x, acc[r][n][2]); acc[r][n][3] = __fmaf_rn(d[r][n][3], s.y, acc[r][n][3]);
        }
}
// the scales of the tokens that a lane's accumulators belong to (token i's scale is known to lanes 4i .. 4i+3)
__device__ __forceinline__ float2 scales_of_columns(float scale, int t)
{
    return make_float2(__shfl_sync(0xffffffffu, scale, 8 * t), __shfl_sync(0xffffffffu, scale, 8 * t + 4));
}
#endif

}  // namespace vptq
