// out = x W^T for at most 16 tokens over an e2m1 weight with a power of two for every 32 columns of a row.
//
// Persistent CTAs, one per SM, own consecutive groups of 16 weight rows and take up to PASS of them (a pass) through all columns.  Each of
// the warps takes every eighth (sixteenth) block of KB columns and feeds itself: a ring of stages in shared memory, a stage one block of the
// pass's rows in one TMA box and the tiles of their scales, refilled as soon as it has been read.
// The warp multiplies in FP16 (mma.sync m16n8k16), in which every code is exact: the order of the products inside a block of 32 columns is free, so
// that lane 4g + t holds codes 8t .. 8t + 7 of rows g and g + 8 and of token g, a word that ldmatrix brings and four conversions widen.  A block's 32
// products are exact in FP32; their sum is multiplied by the weight's power of two and added to the sum of all, times the token's, in one fma.
// (Widened to e4m3 by table look-ups in registers the MMAs are half as many, but a look-up takes 18 clocks a word, the conversions 9.  The
// tcgen05 form, tokens in 128 rows, took 12.0 us for 4096 x 4096 and one token: every block waits for its scales' way into TMEM and its MMAs, one after
// the other, in front of 6 us of setting up.)
// The activations, which no other warp of the CTA needs, come straight from global memory, a block ahead.  Where a CTA has one pass, those of 16 bits, of
// at most 8 tokens, are quantized on the way by the rule of fp4_quantize.cu: a token's block is four lanes.  (Otherwise every CTA's work on all of
// them, pass after pass, would take longer than a kernel in front that does it once.)
// At the end of a pass the warps' sums meet in shared memory and are added in warp order: a result does not depend on timing.
// Every wait is bounded; a warp whose wait gives up leaves NaN, and the workspace's status word is set.
#include "fp4.cuh"
#include "fp4_tcgen05.cuh"
#include "tcgen05_ptx.cuh"
#include "tma_2d.cuh"

namespace vptq {

namespace {

using namespace tc;

constexpr int GROUP = 16;                                 // rows of an MMA
constexpr int MAX_STAGES = 8;                             // of a warp
constexpr int SMEM_MAX = 232448;

__host__ __device__ constexpr int part_stride(int groups) { return groups * GROUP + 4; }               // (lanes of different tokens write different banks)
// bytes of a stage: rows of KB / 2 bytes, tiles of KB / 128 times 512
__host__ __device__ constexpr int group_bytes(int KB) { return GROUP * KB / 2; }
__host__ __device__ constexpr int tile_bytes(int KB) { return KB / FP4_TILE_COLS * FP4_TILE_BYTES; }

struct FewParams {
    Fp4Linear L;
    int col_tiles;
    int passes;                // of every CTA
    int stage_groups, stages;  // groups that a stage holds (the largest pass of any CTA), stages of a warp
    int *status;
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
// acc += (d * w) * s for a pair of sums
__device__ __forceinline__ void add_scaled(float &a0, float &a1, float d0, float d1, float w, float s0, float s1)
{
    asm("{\n\t.reg .b64 a, d, w, s;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 d, {%2, %3};\n\tmov.b64 w, {%4, %4};\n\tmov.b64 s, {%5, %6};\n\t"
        "mul.rn.f32x2 d, d, w;\n\tfma.rn.f32x2 a, d, s, a;\n\tmov.b64 {%0, %1}, a;\n\t}" : "+f"(a0), "+f"(a1) : "f"(d0), "f"(d1), "f"(w), "f"(s0), "f"(s1));
}

// A lane's share of a token's KB columns, 8t .. 8t + 7 of each block of 32, as they lie in memory (16-bit values, two to a word) or as codes with
// the scale bytes of four blocks to a word
template <int DT, int KB> struct Raw { uint4 q[KB / 32]; };
template <int KB> struct Raw<VPTQ_DTYPE_E2M1, KB> { uint32_t q[KB / 32], b[KB / 128]; };

// row: the token's, or null for one that is not there (zeros); c: the lane's first column
template <int DT, bool VEC, int KB>
__device__ __forceinline__ void load_block(Raw<DT, KB> &r, int i, const uint8_t *row, int c, int cols)
{
    c += 32 * i;
    if constexpr (DT == VPTQ_DTYPE_E2M1) {
        r.q[i] = row != nullptr && c < cols ? __ldg(reinterpret_cast<const uint32_t *>(row + c / 2)) : 0u;
    } else if constexpr (VEC) {
        r.q[i] = row != nullptr && c < cols ? __ldg(reinterpret_cast<const uint4 *>(row + 2ll * c)) : make_uint4(0, 0, 0, 0);
    } else {
        uint32_t w[4] = {};
#pragma unroll
        for (int k = 0; k < 8; k++)
            if (row != nullptr && c + k < cols) w[k / 2] |= (uint32_t)__ldg(reinterpret_cast<const uint16_t *>(row) + c + k) << (16 * (k & 1));
        r.q[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// a token's block as an MMA operand, and its scale; for a whole warp.  n: columns from the lane's first on that exist.  zero: 0, which the compiler
// does not know: conversions to e2m1 and back with nothing between them came out as zeros (nvcc 12.9).
template <int DT, int KB>
__device__ __forceinline__ float operand_of(const Raw<DT, KB> &r, int i, int n, uint32_t zero, uint32_t (&h)[4])
{
    if constexpr (DT == VPTQ_DTYPE_E2M1) {
        widen(r.q[i], h);
        return scale_of(r.b[i / 4], i & 3);
    } else {
        Eight<DT, true> e;
        e.q = r.q[i];
        const uint32_t m = larger2(larger2(e.q.x & 0x7FFF7FFFu, e.q.y & 0x7FFF7FFFu), larger2(e.q.z & 0x7FFF7FFFu, e.q.w & 0x7FFF7FFFu));
        const uint32_t b = fp4_block_scale(magnitude16<DT>(m));
        float v[8];
        values_of(e, v);
        widen(fp4_codes(v, b, n) ^ zero, h);
        return fp4_scale_value(b);
    }
}

template <int N> struct Count { static constexpr int value = N; };

// map_full: boxes of stage_groups groups, map_less: of one fewer (passes differ by at most one).  VEC: activations are read 16 bytes at a time.
// PASS: groups of a pass at most; NT: eight tokens, or twice that (e2m1 only).
template <int DT, bool VEC, int PASS, int KB, int NT, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, 1)
linear_fp4_few_kernel(const __grid_constant__ CUtensorMap map_full, const __grid_constant__ CUtensorMap map_less, const __grid_constant__ CUtensorMap map_scales,
                      const __grid_constant__ FewParams D)
{
    const Fp4Linear &P = D.L;
    constexpr int GB = group_bytes(KB), TB = tile_bytes(KB), ROW = KB / 2, BLOCKS = KB / 32;
    constexpr int MAX_TILES = (PASS * GROUP + 2 * FP4_TILE_ROWS - GROUP - 1) / FP4_TILE_ROWS;      // that a pass's rows lie in
    extern __shared__ __align__(1024) uint8_t sm[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t stages = (uint32_t)D.stages, codes_bytes = (uint32_t)(D.stage_groups * GB), stage_bytes = codes_bytes + MAX_TILES * TB;
    const uint32_t ring = smem_addr(sm) + (uint32_t)warp * stages * stage_bytes;
    float *part = reinterpret_cast<float *>(sm + WARPS * stages * stage_bytes);
    const int stride = part_stride(D.stage_groups);
    const uint32_t bars = smem_addr(part) + (uint32_t)(WARPS * 8 * NT * stride * 4 + warp * MAX_STAGES * 8);

    // this CTA's groups, in passes of nearly equal size
    const int groups = (P.M + GROUP - 1) / GROUP, kbs = (P.N + KB - 1) / KB;
    const int first = (int)((long long)groups * blockIdx.x / gridDim.x), count = (int)((long long)groups * (blockIdx.x + 1) / gridDim.x) - first;
    const int passes = D.passes, pass_groups = count / passes, larger = count - pass_groups * passes;
    auto pass_begin = [&](int p) { return first + p * pass_groups + min(p, larger); };
    // this warp's loads, in the order it needs them; by one lane
    int load_pass = warp < kbs ? 0 : passes, load_kb = warp, load_group = first, load_groups = pass_begin(1) - first;
    auto load = [&](uint32_t slot) {
        const uint32_t bar = bars + 8 * slot, to = ring + slot * stage_bytes;
        const int tile = load_group * GROUP / FP4_TILE_ROWS, tiles = ((load_group + load_groups) * GROUP - 1) / FP4_TILE_ROWS - tile + 1;
        mbar_expect_tx(bar, (uint32_t)(load_groups * GB + tiles * TB));
        tma_load_2d(to, load_groups == D.stage_groups ? &map_full : &map_less, load_kb * ROW, load_group * GROUP, bar);
#pragma unroll
        for (int i = 0; i < MAX_TILES; i++)
            if (i < tiles) tma_load_2d(to + codes_bytes + i * TB, &map_scales, 0, (tile + i) * D.col_tiles + load_kb * (KB / FP4_TILE_COLS), bar);
    };
    auto next_load = [&]() {
        load_kb += WARPS;
        if (load_kb >= kbs) {
            load_kb = warp;
            load_pass++;
            load_group = pass_begin(load_pass);
            load_groups = pass_begin(load_pass + 1) - load_group;
        }
    };
    if (lane == 0) {
        for (uint32_t s = 0; s < stages; s++) mbar_init(bars + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_launch_dependents();
    pdl_wait();                                           // (weight, scales and activations may all be the preceding kernel's output)
    for (uint32_t s = 0; s < stages && load_pass < passes; s++) {
        if (lane == 0) load(s);
        next_load();
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *D.status = 0;
    __syncwarp();
    uint32_t gave_up = 0;

    const int g = lane >> 2, t = lane & 3;
    // ldmatrix: this lane names row lane % 16 of a group and, of two adjacent blocks, the first (lanes 0..15) or the second; where that block's piece of
    // the row lies is exchanged by the row's place (128- and 64-byte swizzle), for blocks j and j + 1 by j too
    const int mrow = lane & 15, mblock = lane >> 4;
    const uint32_t piece = (uint32_t)(KB == 256 ? mblock ^ (mrow & 7) : mblock ^ (mrow >> 1 & 3)) << 4;
    const long long pitch = (P.N + FP4_BLOCK - 1ll) / FP4_BLOCK * (FP4_BLOCK / 2);
    const int cols = DT == VPTQ_DTYPE_E2M1 ? (int)(2 * pitch) : P.N;
    const uint8_t *xrow[NT];
#pragma unroll
    for (int u = 0; u < NT; u++)
        xrow[u] = 8 * u + g < P.B ? reinterpret_cast<const uint8_t *>(P.x) + (8 * u + g) * (DT == VPTQ_DTYPE_E2M1 ? pitch : 2ll * P.N) : nullptr;
    auto load_scales = [&](Raw<DT, KB> (&x)[NT], int kb) {
        if constexpr (DT == VPTQ_DTYPE_E2M1) {
#pragma unroll
            for (int u = 0; u < NT; u++)
#pragma unroll
                for (int i = 0; i < KB / 128; i++) {
                    const int tile = kb * (KB / 128) + i;
                    x[u].b[i] = xrow[u] != nullptr && tile < D.col_tiles ? __ldg(reinterpret_cast<const uint32_t *>(P.x_scale + (long long)tile * FP4_TILE_BYTES + fp4_scale_at(8 * u + g, 0))) : 0u;
                }
        }
    };
    const int iterations = warp < kbs ? (kbs - warp + WARPS - 1) / WARPS : 0;
    uint32_t slot = 0, parity = 0;
    for (int p = 0; p < passes; p++) {
        const int g0 = pass_begin(p), n_groups = pass_begin(p + 1) - g0;
        Raw<DT, KB> x[NT];
#pragma unroll
        for (int u = 0; u < NT; u++)
#pragma unroll
            for (int i = 0; i < BLOCKS; i++) load_block<DT, VEC, KB>(x[u], i, warp < kbs ? xrow[u] : nullptr, warp * KB + 8 * t, cols);
        load_scales(x, warp);
        float acc[PASS][NT][4] = {};
        uint32_t scale_at[PASS];                          // of a group's row g, from a stage's scales on
#pragma unroll
        for (int r = 0; r < PASS; r++)
            scale_at[r] = ((g0 + r) * GROUP / FP4_TILE_ROWS - g0 * GROUP / FP4_TILE_ROWS) * TB + fp4_scale_at((g0 + r) * GROUP % FP4_TILE_ROWS, 0) + g * 16;
#pragma unroll 1
        for (int it = 0, kb = warp; it < iterations; it++, kb += WARPS) {
            const uint32_t stage = ring + slot * stage_bytes;
            Raw<DT, KB> next[NT];                         // (e2m1: the next block's scales, whose words all of this one's blocks need)
            load_scales(next, kb + WARPS);
            bool waited = false;
#pragma unroll
            for (int j = 0; j < BLOCKS; j += 2) {
                uint32_t h[NT][2][4];
                float2 s[NT][2];
#pragma unroll
                for (int u = 0; u < NT; u++)
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const float own = operand_of<DT, KB>(x[u], j + i, P.N - (kb * KB + 32 * (j + i) + 8 * t), D.zero, h[u][i]);
                        s[u][i] = make_float2(__shfl_sync(0xffffffffu, own, 8 * t), __shfl_sync(0xffffffffu, own, 8 * t + 4));      // of tokens 2t, 2t + 1
                        load_block<DT, VEC, KB>(x[u], j + i, it + 1 < iterations ? xrow[u] : nullptr, (kb + WARPS) * KB + 8 * t, cols);
                    }
                if (!waited) mbar_wait_within(bars + 8 * slot, parity, D.wait_limit, gave_up);
                waited = true;
                const uint32_t matrices = stage + mrow * ROW + (piece ^ 16 * j), scales = stage + codes_bytes + j / 4 * FP4_TILE_BYTES;
                // R groups from r0 on
                auto multiply = [&](auto count, int r0) {
                    constexpr int R = decltype(count)::value;
                    uint32_t w[R][4], sw[R][2];
#pragma unroll
                    for (int r = 0; r < R; r++) {
                        load_matrices(w[r], matrices + (r0 + r) * GB);
                        sw[r][0] = load_shared(scales + scale_at[r0 + r]);         // of rows g and g + 8
                        sw[r][1] = load_shared(scales + scale_at[r0 + r] + 8 * 16);
                    }
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        uint32_t a[R][4], c[R][4];
                        float d[R][NT][4] = {};
#pragma unroll
                        for (int r = 0; r < R; r++) {
                            widen(w[r][2 * i], a[r]);
                            widen(w[r][2 * i + 1], c[r]);
                        }
                        // step by step over all pairs: the two MMAs of a pair wait for one another
#pragma unroll
                        for (int k = 0; k < 2; k++)
#pragma unroll
                            for (int r = 0; r < R; r++)
#pragma unroll
                                for (int u = 0; u < NT; u++) mma_f16(d[r][u], a[r][2 * k], c[r][2 * k], a[r][2 * k + 1], c[r][2 * k + 1], h[u][i][2 * k], h[u][i][2 * k + 1]);
#pragma unroll
                        for (int r = 0; r < R; r++) {
                            const float f0 = scale_of(sw[r][0], j % 4 + i), f1 = scale_of(sw[r][1], j % 4 + i);
#pragma unroll
                            for (int u = 0; u < NT; u++) {
                                add_scaled(acc[r0 + r][u][0], acc[r0 + r][u][1], d[r][u][0], d[r][u][1], f0, s[u][i].x, s[u][i].y);
                                add_scaled(acc[r0 + r][u][2], acc[r0 + r][u][3], d[r][u][2], d[r][u][3], f1, s[u][i].x, s[u][i].y);
                            }
                        }
                    }
                };
#pragma unroll
                for (int r0 = 0; r0 < PASS; r0 += 2) {
                    if (r0 + 1 < n_groups) multiply(Count<2>{}, r0);
                    else if (r0 < n_groups) multiply(Count<1>{}, r0);
                }
            }
            if constexpr (DT == VPTQ_DTYPE_E2M1)
#pragma unroll
                for (int u = 0; u < NT; u++)
#pragma unroll
                    for (int i = 0; i < KB / 128; i++) x[u].b[i] = next[u].b[i];
            __syncwarp();                                 // every lane has read the stage
            if (load_pass < passes && !__any_sync(0xffffffffu, gave_up != 0)) {
                if (lane == 0) load(slot);
                next_load();
            }
            if (++slot == stages) { slot = 0; parity ^= 1u; }
        }
        // the warps' sums, in warp order
        if (p > 0) asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory");       // the last pass's have been read
        float *mine = part + warp * 8 * NT * stride;
        const bool lost = __any_sync(0xffffffffu, gave_up != 0);      // (every lane's sums hold products of all lanes' operands)
#pragma unroll
        for (int r = 0; r < PASS; r++) {
            if (r >= n_groups) break;
#pragma unroll
            for (int u = 0; u < NT; u++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    mine[(8 * u + 2 * t + (i & 1)) * stride + r * GROUP + g + 8 * (i >> 1)] = lost ? __int_as_float(0x7FFFFFFF) : acc[r][u][i];
        }
        asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory");
        const int rows = n_groups * GROUP, m0 = g0 * GROUP;
        for (int i = threadIdx.x; i < P.B * rows; i += 32 * WARPS) {
            const int token = i / rows, m = i % rows;
            if (m0 + m >= P.M) continue;
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; w++) sum += part[(w * 8 * NT + token) * stride + m];
            if (!(fabsf(sum) < __int_as_float(0x7F800000))) sum = __int_as_float(0x7FFFFFFF);           // (a weight's scale that is NaN)
            store_out(P.out, (long long)token * P.M + m0 + m, sum, P.out_dtype);
        }
    }
    if (gave_up) {
        let_copies_land();
        atomicExch(D.status, VPTQ_E_TIMEOUT);                          // (long after the word was cleared)
    }
}

template <int DT, bool VEC, int PASS, int KB, int NT, int WARPS>
cudaError_t run(const Fp4Linear &P, int *status, cudaStream_t st)
{
    constexpr int MAX_TILES = (PASS * GROUP + 2 * FP4_TILE_ROWS - GROUP - 1) / FP4_TILE_ROWS;
    const long long pitch = fp4_row_bytes(P.N);
    const int groups = ceil_div(P.M, GROUP), sms = device_sm_count(), grid = groups < sms ? groups : sms, kbs = ceil_div(P.N, KB);
    const int most = ceil_div(groups, grid);              // groups of a CTA
    FewParams D;
    D.L = P;
    D.col_tiles = ceil_div(P.N, FP4_TILE_COLS);
    D.passes = ceil_div(most, PASS);
    D.stage_groups = ceil_div(most, D.passes);
    D.status = status;
    D.zero = 0;
    D.wait_limit = wait_limit();
    const int stage = D.stage_groups * group_bytes(KB) + MAX_TILES * tile_bytes(KB);
    const int fixed = WARPS * 8 * NT * part_stride(D.stage_groups) * 4 + WARPS * MAX_STAGES * 8;
    D.stages = (SMEM_MAX - fixed) / (WARPS * stage);
    if (D.stages > MAX_STAGES) D.stages = MAX_STAGES;
    const long long loads = (long long)ceil_div(kbs, WARPS) * D.passes;
    if (D.stages > loads) D.stages = (int)loads;
    const int smem = D.stages * WARPS * stage + fixed;
    CUtensorMap map[2], map_scales;
    for (int i = 0; i < 2; i++) {
        const int rows = GROUP * (D.stage_groups - i > 0 ? D.stage_groups - i : 1);
        if (!encode_tensor_map(&map[i], CU_TENSOR_MAP_DATA_TYPE_UINT8, P.w, pitch, P.M, pitch, 0, 0, KB / 2, rows, 1, KB == 256 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B))
            return cudaErrorNotSupported;
    }
    if (!encode_tensor_map(&map_scales, CU_TENSOR_MAP_DATA_TYPE_UINT32, P.w_scale, FP4_TILE_BYTES / 4, (uint64_t)(fp4_scale_bytes(P.M, P.N) / FP4_TILE_BYTES), FP4_TILE_BYTES, 0, 0,
                           FP4_TILE_BYTES / 4, KB / FP4_TILE_COLS, 1, CU_TENSOR_MAP_SWIZZLE_NONE))
        return cudaErrorNotSupported;
    auto kern = linear_fp4_few_kernel<DT, VEC, PASS, KB, NT, WARPS>;
    const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void *>(kern), SMEM_MAX);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(32 * WARPS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = pdl_enabled("linear_fp4") ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, map[0], map[1], map_scales, D);
}

// Up to two groups a CTA, in one pass: 16-bit activations are quantized on the way.  More, in passes of four: blocks of half as many columns, so that
// two stages a warp fit.
template <int DT, bool VEC, int NT>
cudaError_t run_small(const Fp4Linear &P, int *status, cudaStream_t st) { return run<DT, VEC, 2, 256, NT, 16>(P, status, st); }
template <int NT>
cudaError_t run_large(const Fp4Linear &P, int *status, cudaStream_t st) { return run<VPTQ_DTYPE_E2M1, true, 4, 128, NT, 16>(P, status, st); }
bool small(int M) { return ceil_div(M, GROUP) <= 2 * device_sm_count(); }

}  // namespace

bool linear_fp4_few_quantizes(int M, int B) { return B <= 8 && small(M); }

cudaError_t launch_linear_fp4_few(const Fp4Linear &P, int *status, cudaStream_t st)
{
    if (!small(P.M)) return P.B > 8 ? run_large<2>(P, status, st) : run_large<1>(P, status, st);
    const bool vec = P.N % 8 == 0 && (reinterpret_cast<uintptr_t>(P.x) & 15u) == 0;
    if (P.x_dtype == VPTQ_DTYPE_E2M1) return P.B > 8 ? run_small<VPTQ_DTYPE_E2M1, true, 2>(P, status, st) : run_small<VPTQ_DTYPE_E2M1, true, 1>(P, status, st);
    if (P.x_dtype == VPTQ_DTYPE_BF16) return vec ? run_small<VPTQ_DTYPE_BF16, true, 1>(P, status, st) : run_small<VPTQ_DTYPE_BF16, false, 1>(P, status, st);
    return vec ? run_small<VPTQ_DTYPE_FP16, true, 1>(P, status, st) : run_small<VPTQ_DTYPE_FP16, false, 1>(P, status, st);
}

}  // namespace vptq
