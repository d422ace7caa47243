// out = x W^T for at most 8 tokens in 16 bits over a small e2m1 weight: the activations are quantized on the way, in one kernel.
//
// CTAs, one per SM, own one or two consecutive groups of 16 weight rows.  Each of the 16 warps takes 256 columns of them and feeds itself: one TMA box
// of the CTA's rows (128-byte swizzle) and the tiles of their scales.
// The warp multiplies in FP16 (mma.sync m16n8k16), in which every code is exact: the order of the products inside a block of 32 columns is free, so
// that lane 4g + t holds codes 8t .. 8t + 7 of rows g and g + 8 and of token g, a word that ldmatrix brings and four conversions widen.  A block's 32
// products are exact in FP32; their sum is multiplied by the weight's power of two and added to the sum of all, times the token's, in one fma.
// The activations, which no other warp of the CTA needs, come straight from global memory and are quantized by the rule of fp4_quantize.cu: a
// token's block is four lanes.  At the end the warps' sums meet in shared memory and are added in warp order.
// 4096 x 4096, one token, 5.6 us, weights out of HBM in a graph: launch, first reads and a warp's eight dependent steps.  No pipe is used up (issue slots
// 49 % busy, the integer pipe 41 %, for which a word's widening is 7 instructions, four conversions and the bytes' ways to them).
// Larger weights go to linear_fp4_tcgen05.cu behind a quantizing kernel, whose products cost no instructions.  A form of this kernel that went over them
// in passes, the integer pipe its bound, took 36 us for 28672 x 8192 and one token, that one 22.
// Every wait is bounded; a warp whose wait gives up leaves NaN.
#include "fp4.cuh"
#include "fp4_tcgen05.cuh"
#include "tcgen05_ptx.cuh"
#include "tma_2d.cuh"

namespace vptq {

namespace {

using namespace tc;

constexpr int GROUP = 16, GROUPS = 2;                     // rows of an MMA, groups of a CTA at most
constexpr int WARPS = 16;
constexpr int KB = 256, ROW = KB / 2, BLOCKS = KB / FP4_BLOCK, CHUNKS = KB / FP4_TILE_COLS;
constexpr int GROUP_BYTES = GROUP * ROW, TILES = 2;       // tiles of scales that a CTA's rows may lie in
constexpr int STAGE_BYTES = GROUPS * GROUP_BYTES + TILES * CHUNKS * FP4_TILE_BYTES;
constexpr int STRIDE = GROUPS * GROUP + 4;                // of a token's sums (lanes of different tokens write different banks)
constexpr int MAX_COLS = WARPS * KB;                      // a block a warp
constexpr int SMEM = WARPS * STAGE_BYTES;
static_assert(8 * STRIDE * 4 <= STAGE_BYTES, "a warp's sums take its operands' place");

struct FewParams {
    Fp4Linear L;
    int stage_groups;                         // the most of any CTA
    uint32_t zero;
    unsigned long long wait_limit;
};

__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t a)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a));
}
__device__ __forceinline__ uint32_t load_shared(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
// eight codes as FP16
__device__ __forceinline__ void widen(uint32_t q, uint32_t (&h)[4])
{
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\tcvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(q));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Byte i of a word of scales as a power of two; 0 is 2^-127, and 255 an infinity: what it is multiplied into is no number, or is told by that.
__device__ __forceinline__ float scale_of(uint32_t w, int i)
{
    const uint32_t bits = (i == 3 ? w >> 1 : w << (23 - 8 * i)) & 0x7F800000u;
    return __uint_as_float(max(bits, 0x00400000u));
}

// Eight columns from c on of a token's row (null: a token that is not there) as they lie in memory, zeros beyond `cols`
template <bool VEC>
__device__ __forceinline__ uint4 load_columns(const uint8_t *row, int c, int cols)
{
    if constexpr (VEC) return row != nullptr && c < cols ? __ldg(reinterpret_cast<const uint4 *>(row + 2ll * c)) : make_uint4(0, 0, 0, 0);
    uint32_t w[4] = {};
#pragma unroll
    for (int k = 0; k < 8; k++)
        if (row != nullptr && c + k < cols) w[k / 2] |= (uint32_t)__ldg(reinterpret_cast<const uint16_t *>(row) + c + k) << (16 * (k & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// a token's block as an MMA operand, and its scale; for a whole warp.  n: columns from the lane's first on that exist.  zero: 0, which the compiler
// does not know: conversions to e2m1 and back with nothing between them came out as zeros (nvcc 12.9).
// A block's 32 products add up to at most 1152, times the weight's power of two at most 2^127: so that this does not overflow where the token's
// power makes it small again, the operand is taken 2^11 smaller and its scale as much larger (all of it exact: the smallest step is 2^-140), unless
// that scale is itself so large that the result overflows.
template <int DT>
__device__ __forceinline__ float operand_of(uint4 q, int n, uint32_t zero, uint32_t (&h)[4])
{
    Eight<DT, true> e;
    e.q = q;
    const uint32_t m = larger2(larger2(q.x & 0x7FFF7FFFu, q.y & 0x7FFF7FFFu), larger2(q.z & 0x7FFF7FFFu, q.w & 0x7FFF7FFFu));
    const uint32_t b = fp4_block_scale(magnitude16<DT>(m));
    float v[8];
    values_of(e, v);
    widen(fp4_codes(v, b, n) ^ zero, h);
    const bool down = b < 243u;
    const __half2 by = __half2half2(__ushort_as_half(down ? 0x1000 : 0x3C00));         // 2^-11 or 1
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const __half2 p = __hmul2(*reinterpret_cast<const __half2 *>(&h[i]), by);
        h[i] = *reinterpret_cast<const uint32_t *>(&p);
    }
    return __uint_as_float(b == 255u ? 0x7FFFFFFFu : (b + (down ? 11u : 0u)) << 23);
}

// map_full: boxes of stage_groups groups, map_less: of one fewer (CTAs differ by at most one).  VEC: activations are read 16 bytes at a time.
template <int DT, bool VEC>
__global__ void __launch_bounds__(32 * WARPS, 1)
linear_fp4_few_kernel(const __grid_constant__ CUtensorMap map_full, const __grid_constant__ CUtensorMap map_less, const __grid_constant__ CUtensorMap map_scales,
                      const __grid_constant__ FewParams D)
{
    const Fp4Linear &P = D.L;
    extern __shared__ __align__(1024) uint8_t sm[];
    __shared__ __align__(8) uint64_t barriers[WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t stage = smem_addr(sm) + (uint32_t)(warp * STAGE_BYTES), bar = smem_addr(barriers + warp);

    const int groups = (P.M + GROUP - 1) / GROUP, kbs = (P.N + KB - 1) / KB;
    const int g0 = (int)((long long)groups * blockIdx.x / gridDim.x), n_groups = (int)((long long)groups * (blockIdx.x + 1) / gridDim.x) - g0;
    const int tile0 = g0 * GROUP / FP4_TILE_ROWS, tiles = ((g0 + n_groups) * GROUP - 1) / FP4_TILE_ROWS - tile0 + 1;
    const bool any = warp < kbs;                          // (the same for the warp's lanes)
    if (lane == 0) {
        mbar_init(bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_launch_dependents();
    pdl_wait();                                           // (weight, scales and activations may all be the preceding kernel's output)
    if (lane == 0 && any) {
        mbar_expect_tx(bar, (uint32_t)(n_groups * GROUP_BYTES + tiles * CHUNKS * FP4_TILE_BYTES));
        tma_load_2d(stage, n_groups == D.stage_groups ? &map_full : &map_less, warp * ROW, g0 * GROUP, bar);
        // (zeros beyond a row's last tile, as the codes there: what follows in memory is the next 128 rows', and 0 * NaN is not 0)
        for (int i = 0; i < tiles; i++)
            tma_load_3d(stage + GROUPS * GROUP_BYTES + i * CHUNKS * FP4_TILE_BYTES, &map_scales, 0, warp * CHUNKS, tile0 + i, bar);
    }
    __syncwarp();
    uint32_t gave_up = 0;

    const int g = lane >> 2, t = lane & 3;
    // ldmatrix: this lane names row lane % 16 of a group and, of two adjacent blocks, the first (lanes 0..15) or the second; where that block's piece of
    // the row lies is exchanged by the row's place among eight, for blocks j and j + 1 by j too
    const int mrow = lane & 15;
    const uint32_t piece = (uint32_t)(lane >> 4 ^ (mrow & 7)) << 4;
    uint32_t scale_at[GROUPS];                            // of a group's row g, from a stage's scales on
#pragma unroll
    for (int r = 0; r < GROUPS; r++)
        scale_at[r] = ((g0 + r) * GROUP / FP4_TILE_ROWS - tile0) * CHUNKS * FP4_TILE_BYTES + fp4_scale_at((g0 + r) * GROUP % FP4_TILE_ROWS, 0) + g * 16;
    const uint8_t *xrow = g < P.B ? reinterpret_cast<const uint8_t *>(P.x) + g * 2ll * P.N : nullptr;
    uint4 x[BLOCKS];
#pragma unroll
    for (int i = 0; i < BLOCKS; i++) x[i] = load_columns<VEC>(xrow, warp * KB + 32 * i + 8 * t, P.N);
    float acc[GROUPS][4] = {};
    if (any) {
#pragma unroll
        for (int j = 0; j < BLOCKS; j += 2) {
            uint32_t h[2][4];
            float2 s[2];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const float own = operand_of<DT>(x[j + i], P.N - (warp * KB + 32 * (j + i) + 8 * t), D.zero, h[i]);
                s[i] = make_float2(__shfl_sync(0xffffffffu, own, 8 * t), __shfl_sync(0xffffffffu, own, 8 * t + 4));          // of tokens 2t, 2t + 1
            }
            if (j == 0) mbar_wait_within(bar, 0, D.wait_limit, gave_up);
            const uint32_t matrices = stage + mrow * ROW + (piece ^ 16 * j), scales = stage + GROUPS * GROUP_BYTES + j / 4 * FP4_TILE_BYTES;
            // (a second group that the CTA does not have is multiplied all the same, and dropped)
            uint32_t w[GROUPS][4], sw[GROUPS][2];
#pragma unroll
            for (int r = 0; r < GROUPS; r++) {
                load_matrices(w[r], matrices + r * GROUP_BYTES);
                sw[r][0] = load_shared(scales + scale_at[r]);                  // of rows g and g + 8
                sw[r][1] = load_shared(scales + scale_at[r] + 8 * 16);
            }
#pragma unroll
            for (int i = 0; i < 2; i++) {
                uint32_t a[GROUPS][4], c[GROUPS][4];
                float d[GROUPS][4] = {};
#pragma unroll
                for (int r = 0; r < GROUPS; r++) {
                    widen(w[r][2 * i], a[r]);
                    widen(w[r][2 * i + 1], c[r]);
                }
#pragma unroll
                for (int k = 0; k < 4; k += 2)
#pragma unroll
                    for (int r = 0; r < GROUPS; r++) mma_f16(d[r], a[r][k], c[r][k], a[r][k + 1], c[r][k + 1], h[i][k], h[i][k + 1]);
#pragma unroll
                for (int r = 0; r < GROUPS; r++) {
                    const float f0 = scale_of(sw[r][0], j % 4 + i), f1 = scale_of(sw[r][1], j % 4 + i);
                    acc[r][0] = __fmaf_rn(d[r][0] * f0, s[i].x, acc[r][0]); acc[r][1] = __fmaf_rn(d[r][1] * f0, s[i].y, acc[r][1]);
                    acc[r][2] = __fmaf_rn(d[r][2] * f1, s[i].x, acc[r][2]); acc[r][3] = __fmaf_rn(d[r][3] * f1, s[i].y, acc[r][3]);
                }
            }
        }
    }
    // the warps' sums, in warp order (each where its operands were, which all its lanes have read)
    __syncwarp();
    float *mine = reinterpret_cast<float *>(sm + warp * STAGE_BYTES);
    const bool lost = __any_sync(0xffffffffu, gave_up != 0);          // (every lane's sums hold products of all lanes' operands)
    if (lost) let_copies_land();                                      // (before anything else lies in their place)
#pragma unroll
    for (int r = 0; r < GROUPS; r++)
#pragma unroll
        for (int i = 0; i < 4; i++) mine[(2 * t + (i & 1)) * STRIDE + r * GROUP + g + 8 * (i >> 1)] = lost ? __int_as_float(0x7FFFFFFF) : acc[r][i];
    __syncthreads();
    const int rows = n_groups * GROUP, m0 = g0 * GROUP;
    for (int i = threadIdx.x; i < P.B * rows; i += 32 * WARPS) {
        const int token = i / rows, m = i % rows;
        if (m0 + m >= P.M) continue;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; w++) sum += reinterpret_cast<const float *>(sm + w * STAGE_BYTES)[token * STRIDE + m];
        if (!(fabsf(sum) < __int_as_float(0x7F800000))) sum = __int_as_float(0x7FFFFFFF);               // (a weight's scale that is NaN)
        store_out(P.out, (long long)token * P.M + m0 + m, sum, P.out_dtype);
    }
}

template <int DT, bool VEC>
cudaError_t run(const Fp4Linear &P, cudaStream_t st)
{
    const long long pitch = fp4_row_bytes(P.N);
    const int groups = ceil_div(P.M, GROUP), sms = device_sm_count(), grid = groups < sms ? groups : sms;
    FewParams D;
    D.L = P;
    D.stage_groups = ceil_div(groups, grid);
    D.zero = 0;
    D.wait_limit = wait_limit();
    CUtensorMap map[2], map_scales;
    for (int i = 0; i < 2; i++) {
        const int rows = GROUP * (D.stage_groups - i > 0 ? D.stage_groups - i : 1);
        if (!encode_tensor_map(&map[i], CU_TENSOR_MAP_DATA_TYPE_UINT8, P.w, pitch, P.M, pitch, 0, 0, ROW, rows, 1, CU_TENSOR_MAP_SWIZZLE_128B)) return cudaErrorNotSupported;
    }
    const uint64_t col_tiles = (uint64_t)ceil_div(P.N, FP4_TILE_COLS), row_tiles = (uint64_t)ceil_div(P.M, FP4_TILE_ROWS);
    if (!encode_tensor_map(&map_scales, CU_TENSOR_MAP_DATA_TYPE_UINT32, P.w_scale, FP4_TILE_BYTES / 4, col_tiles, FP4_TILE_BYTES, row_tiles, col_tiles * FP4_TILE_BYTES,
                           FP4_TILE_BYTES / 4, CHUNKS, 1, CU_TENSOR_MAP_SWIZZLE_NONE))
        return cudaErrorNotSupported;
    auto kern = linear_fp4_few_kernel<DT, VEC>;
    const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void *>(kern), SMEM);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(32 * WARPS);
    cfg.dynamicSmemBytes = SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = pdl_enabled("linear_fp4") ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, map[0], map[1], map_scales, D);
}

}  // namespace

// One launch instead of two, and 2 to 3 us less of the host's time.  In a graph, this kernel / the two, weights out of HBM, one token:
//   512 rows:   128 columns 2.8 / 3.7 us, 1024 2.9 / 4.5, 2048 3.4 / 4.6, 4096 4.5 / 4.9
//   4096 rows:  128 columns 2.9 / 3.5, 1024 3.2 / 5.0, 2048 4.1 / 6.0, 4096 5.6 / 7.5 (8 tokens 6.6 / 7.6)
//   4736 rows (32 an SM):  4096 columns 5.8 / 8.1
// A warp's columns are one step of loads: more than 4096 would take a second, while the gain is already shrinking (64 rows of 4096, 8 tokens: 4.7 / 4.5).
// Rows that are no multiples of 16 bytes, read value by value, would take longer than the other launch.
bool linear_fp4_few_takes(int M, int N, int B, int x_dtype)
{
    return x_dtype != VPTQ_DTYPE_E2M1 && B <= 8 && N <= MAX_COLS && N % 8 == 0 && ceil_div(M, GROUP) <= GROUPS * device_sm_count();
}

cudaError_t launch_linear_fp4_few(const Fp4Linear &P, cudaStream_t st)
{
    const bool vec = (reinterpret_cast<uintptr_t>(P.x) & 15u) == 0;
    if (P.x_dtype == VPTQ_DTYPE_BF16) return vec ? run<VPTQ_DTYPE_BF16, true>(P, st) : run<VPTQ_DTYPE_BF16, false>(P, st);
    return vec ? run<VPTQ_DTYPE_FP16, true>(P, st) : run<VPTQ_DTYPE_FP16, false>(P, st);
}

}  // namespace vptq
