// out = x W^T for at most 8 tokens over an e4m3 weight with 128 x 128 block scales.
//
// Persistent CTAs, one per SM, own consecutive groups of 16 output rows and take up to PASS of them (a pass) through all columns.  Each of
// the 8 or 16 warps takes every eighth (sixteenth) run of 128-column blocks and feeds itself: a ring of stages in shared memory, a stage one run of the
// pass's rows in one TMA box (128-byte swizzle), refilled as soon as it has been read.  A run is as many blocks as make 8 KB (one where
// rows are no multiple of 128 bytes): fewer copies and waits (4096 x 4096, one token in 16 bits, 6.8 us; a block at a time 7.2).  The
// activations, which no other warp of the CTA needs, come straight from global memory, two blocks ahead.  (A ring for the whole CTA
// filled by a warp of its own took 11.0 us.)  The scales are fetched for 32 (the
// weight's) or 4 blocks (the tokens') at a time, one to a lane.
// The warp multiplies (fp8_mma.cuh) and keeps FP32 sums of all the pass's rows.  16-bit activations are quantized on the way, by the
// same rule as vptq_fp8_quantize: the four lanes that hold a token's block find its maximum with two shuffles, and all the pass's rows
// share that work.  At the end of a pass the warps' sums meet in shared memory and are added in warp order: a result does not depend on
// timing.
// Large weights are bound by HBM, M * N bytes (28672 x 8192 40.4 us, 5.8 TB/s); small ones by what a warp does for a block, one step
// after the other: 1000 to 1900 clocks.
// Every wait is bounded; a warp whose wait gives up leaves NaN from there on.
#include "fp8_mma.cuh"
#include "tcgen05_ptx.cuh"
#include "tma_2d.cuh"

namespace vptq {

namespace {

using namespace tc;

constexpr int GROUP = 16;                                 // rows of an MMA
constexpr int GROUP_BYTES = GROUP * FP8_BLOCK;
constexpr int MAX_STAGES = 8;                             // of a warp
constexpr int SMEM_MAX = 232448;

__host__ __device__ constexpr int part_stride(int groups) { return groups * GROUP + 4; }               // (lanes of different tokens write different banks)

struct DecodeParams {
    Fp8Linear L;
    int passes;                // of every CTA
    int stage_groups, stages;  // groups that a stage holds (the largest pass of any CTA), stages of a warp
    int run_shift;             // log2 of a stage's blocks
    unsigned long long wait_limit;
};

__device__ __forceinline__ uint4 load_shared16(uint32_t a)
{
    uint4 q;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(a));
    return q;
}

// map_full: boxes of stage_groups groups, map_less: of one fewer (passes differ by at most one); RUNS: the maps have the blocks as a third
// dimension.  VEC: activations are read 16 bytes at a time.  PASS: groups of a pass at most.
template <int DT, bool VEC, int PASS, bool RUNS, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, 1)
linear_fp8_decode_kernel(const __grid_constant__ CUtensorMap map_full, const __grid_constant__ CUtensorMap map_less, const __grid_constant__ DecodeParams D)
{
    constexpr int BATCH = PASS < 4 ? 2 : 3;    // groups whose operands a warp holds, and whose MMAs it has under way, at a time
    const Fp8Linear &P = D.L;
    extern __shared__ __align__(1024) uint8_t sm[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, run_shift = RUNS ? D.run_shift : 0, run = 1 << run_shift;
    const uint32_t stages = (uint32_t)D.stages, block_bytes = (uint32_t)(D.stage_groups * GROUP_BYTES), stage_bytes = block_bytes * run;
    const uint32_t ring = smem_addr(sm) + (uint32_t)warp * stages * stage_bytes;
    float *part = reinterpret_cast<float *>(sm + WARPS * stages * stage_bytes);
    const int stride = part_stride(D.stage_groups);
    const uint32_t bars = smem_addr(part) + (uint32_t)(WARPS * 8 * stride * 4 + warp * MAX_STAGES * 8);

    // this CTA's groups, in passes of nearly equal size
    const int groups = (P.M + GROUP - 1) / GROUP, kbs = (P.N + FP8_BLOCK - 1) / FP8_BLOCK, runs = (kbs + run - 1) >> run_shift;
    const int first = (int)((long long)groups * blockIdx.x / gridDim.x), count = (int)((long long)groups * (blockIdx.x + 1) / gridDim.x) - first;
    const int passes = D.passes;
    // (the first passes are a group larger where they do not come out even; no divisions in the loop below: they took 2000 clocks a stage)
    const int pass_groups = count / passes, larger = count - pass_groups * passes;
    auto pass_begin = [&](int p) { return first + p * pass_groups + min(p, larger); };
    // this warp's loads, in the order it needs them; by one lane
    int load_pass = warp < runs ? 0 : passes, load_run = warp, load_row = first * GROUP, load_groups = pass_begin(1) - first;
    auto load = [&](uint32_t slot) {
        const uint32_t bar = bars + 8 * slot, to = ring + slot * stage_bytes;
        const CUtensorMap *map = load_groups == D.stage_groups ? &map_full : &map_less;
        mbar_expect_tx(bar, (uint32_t)(load_groups * GROUP_BYTES * run));
        if (RUNS) tma_load_3d(to, map, 0, load_row, load_run * run, bar);
        else tma_load_2d(to, map, load_run * FP8_BLOCK, load_row, bar);
    };
    auto next_load = [&]() {
        load_run += WARPS;
        if (load_run >= runs) {
            load_run = warp;
            load_pass++;
            load_row = pass_begin(load_pass) * GROUP;
            load_groups = pass_begin(load_pass + 1) - pass_begin(load_pass);
        }
    };
    if (lane == 0) {
        for (uint32_t s = 0; s < stages; s++) mbar_init(bars + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_launch_dependents();
    // (weight, scales and activations may all be the preceding kernel's output; weights ahead of the wait would save 0.2 us of a call)
    pdl_wait();
    for (uint32_t s = 0; s < stages && load_pass < passes; s++) {
        if (lane == 0) load(s);
        next_load();
    }
    __syncwarp();
    uint32_t gave_up = 0;

    const int g = lane >> 2, t = lane & 3;
    const int row = (g >> 1) | ((g & 1) << 2);            // the MMA's row g is this row of a box: a quarter warp's reads then fall into different banks
    const uint32_t at0 = (uint32_t)(row * FP8_BLOCK + ((t ^ row) << 4)), at1 = (uint32_t)(row * FP8_BLOCK + (((t + 4) ^ row) << 4));
    const long long pitch = (P.N + 15ll) / 16 * 16;
    const int cols = DT == VPTQ_DTYPE_E4M3 ? (int)pitch : P.N;
    const uint8_t *xrow = g < P.B ? reinterpret_cast<const uint8_t *>(P.x) + (DT == VPTQ_DTYPE_E4M3 ? g * pitch : (long long)g * P.N * 2) : nullptr;
    // this warp's blocks in order: block i of them is block i % run of its run i / run
    auto next_block = [&](int kb) {
        kb++;
        if ((kb & (run - 1)) == 0) kb += (WARPS - 1) << run_shift;
        return kb;
    };
    int iterations = 0;                                   // blocks of a pass
    if (warp < runs) {
        const int mine = (runs - warp + WARPS - 1) / WARPS;                    // runs; the last one of all may be short
        iterations = mine * run - ((warp + (mine - 1) * WARPS) == runs - 1 ? runs * run - kbs : 0);
    }
    uint32_t slot = 0, parity = 0;
    for (int p = 0; p < passes; p++) {
        const int g0 = pass_begin(p), n_groups = pass_begin(p + 1) - g0;
        // the pass's rows lie in one 128-row block of the weight, or in two from group `second` on
        const int block = g0 * GROUP / FP8_BLOCK, last = (P.M - 1) / FP8_BLOCK, second = FP8_BLOCK / GROUP - g0 % (FP8_BLOCK / GROUP);
        const float *ws0 = P.w_scale + (long long)block * kbs, *ws1 = P.w_scale + (long long)min(block + 1, last) * kbs;
        // scales of the warp's blocks: the weight's of its blocks 32 j + lane, a token's of 4 j + t in its four lanes
        auto block_of = [&](int i) { return ((warp + (i >> run_shift) * WARPS) << run_shift) + (i & (run - 1)); };
        auto weight_scales = [&](const float *ws, int i) { return i + lane < iterations ? __ldg(ws + block_of(i + lane)) : 0.f; };
        auto token_scale = [&](int i) { return DT == VPTQ_DTYPE_E4M3 && g < P.B && i + t < iterations ? __ldg(P.x_scale + (long long)g * kbs + block_of(i + t)) : 0.f; };
        float w0 = weight_scales(ws0, 0), w1 = weight_scales(ws1, 0), ts = 0.f, ts_next = token_scale(0);
        TokenRaw<DT, VEC> x, x_next;
        int kb_ahead = warp * run;                        // the next block whose activations are fetched
        auto fetch = [&](TokenRaw<DT, VEC> &to) {
            to = load_token<DT, VEC>(kb_ahead < kbs ? xrow : nullptr, t, kb_ahead, cols);
            kb_ahead = next_block(kb_ahead);
        };
        fetch(x);
        fetch(x_next);
        float acc[(PASS + BATCH - 1) / BATCH * BATCH][1][4] = {};
        int in_run = 0;
#pragma unroll 1
        for (int i = 0; i < iterations; i++) {
            if ((i & 31) == 0 && i > 0) { w0 = weight_scales(ws0, i); w1 = weight_scales(ws1, i); }
            if (DT == VPTQ_DTYPE_E4M3 && (i & 3) == 0) { ts = ts_next; ts_next = token_scale(i + 4); }
            const float c0 = __shfl_sync(0xffffffffu, w0, i & 31), c1 = __shfl_sync(0xffffffffu, w1, i & 31);
            const TokenFrag b[1] = {quantize_token<DT, VEC>(x, __shfl_sync(0xffffffffu, ts, (lane & ~3) | (i & 3)))};
            const float2 s = scales_of_columns(b[0].scale, t);
            x = x_next;
            fetch(x_next);
            const uint32_t stage = ring + slot * stage_bytes + (uint32_t)(in_run * n_groups * GROUP_BYTES);
            if (in_run == 0) mbar_wait_within(bars + 8 * slot, parity, D.wait_limit, gave_up);
            // (groups that the pass does not have are multiplied with whatever lies behind its own, and dropped)
#pragma unroll
            for (int r0 = 0; r0 < PASS; r0 += BATCH) {
                if (r0 >= n_groups) break;
                WeightFrag a[BATCH];
#pragma unroll
                for (int r = 0; r < BATCH; r++) {
                    const uint32_t box = stage + (r0 + r) * GROUP_BYTES;
                    a[r].q[0][0] = load_shared16(box + at0); a[r].q[1][0] = load_shared16(box + 8 * FP8_BLOCK + at0);
                    a[r].q[0][1] = load_shared16(box + at1); a[r].q[1][1] = load_shared16(box + 8 * FP8_BLOCK + at1);
                }
                block_products<BATCH, 1>(&acc[r0], a, b, [&](int r, int) {
                    const float w = r0 + r < second ? c0 : c1;
                    return make_float2(s.x * w, s.y * w);
                });
            }
            if (++in_run == run || i == iterations - 1) {
                in_run = 0;
                __syncwarp();                             // every lane has read the stage
                if (load_pass < passes && !__any_sync(0xffffffffu, gave_up != 0)) {
                    if (lane == 0) load(slot);
                    next_load();
                }
                if (++slot == stages) { slot = 0; parity ^= 1u; }
            }
        }
        // the warps' sums, in warp order
        if (p > 0) asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory");       // the last pass's have been read
        float *mine = part + warp * 8 * stride;
        const bool lost = __any_sync(0xffffffffu, gave_up != 0);      // (every lane's sums hold products of all lanes' operands)
#pragma unroll
        for (int r = 0; r < PASS; r++) {
            if (r >= n_groups) break;
#pragma unroll
            for (int i = 0; i < 4; i++) mine[(2 * t + (i & 1)) * stride + r * GROUP + row + 8 * (i >> 1)] = lost ? __int_as_float(0x7FFFFFFF) : acc[r][0][i];
        }
        asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory");
        const int rows = n_groups * GROUP, m0 = g0 * GROUP;
        for (int i = threadIdx.x; i < P.B * rows; i += 32 * WARPS) {
            const int token = i / rows, m = i % rows;
            if (m0 + m >= P.M) continue;
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; w++) sum += part[(w * 8 + token) * stride + m];
            store_out(P.out, (long long)token * P.M + m0 + m, sum, P.out_dtype);
        }
    }
    if (gave_up) let_copies_land();
}

template <int DT, bool VEC, int PASS, bool RUNS, int WARPS>
cudaError_t run(const Fp8Linear &P, cudaStream_t st)
{
    const long long pitch = fp8_row_bytes(P.N);
    const int groups = ceil_div(P.M, GROUP), sms = device_sm_count(), grid = groups < sms ? groups : sms, kbs = ceil_div(P.N, FP8_BLOCK);
    const int most = ceil_div(groups, grid);              // groups of a CTA
    DecodeParams D;
    D.L = P;
    D.passes = ceil_div(most, PASS);
    D.stage_groups = ceil_div(most, D.passes);
    D.wait_limit = wait_limit();
    D.run_shift = 0;                                      // up to 8 KB, but something to do for every warp first
    if (RUNS)
        while ((2 << D.run_shift) * D.stage_groups <= 4 && ceil_div(kbs, 2 << D.run_shift) >= WARPS) D.run_shift++;
    const int run = 1 << D.run_shift, stage = D.stage_groups * GROUP_BYTES * run;
    const int fixed = WARPS * 8 * part_stride(D.stage_groups) * 4 + WARPS * MAX_STAGES * 8;
    // (the last stage's reads may run on for up to three groups: into the sums, which are at least as large)
    D.stages = (SMEM_MAX - fixed) / (WARPS * stage);
    if (D.stages > MAX_STAGES) D.stages = MAX_STAGES;
    const int loads = ceil_div(ceil_div(kbs, run), WARPS) * D.passes;
    if (D.stages > loads) D.stages = loads;
    const int smem = D.stages * WARPS * stage + fixed;
    CUtensorMap map[2];
    for (int i = 0; i < 2; i++) {
        const int rows = GROUP * (D.stage_groups - i > 0 ? D.stage_groups - i : 1);
        if (!(RUNS ? encode_tensor_map(&map[i], CU_TENSOR_MAP_DATA_TYPE_UINT8, P.w, FP8_BLOCK, P.M, pitch, kbs, FP8_BLOCK, FP8_BLOCK, rows, run, CU_TENSOR_MAP_SWIZZLE_128B)
                   : encode_tensor_map(&map[i], CU_TENSOR_MAP_DATA_TYPE_UINT8, P.w, pitch, P.M, pitch, 0, 0, FP8_BLOCK, rows, 1, CU_TENSOR_MAP_SWIZZLE_128B)))
            return cudaErrorNotSupported;
    }
    auto kern = linear_fp8_decode_kernel<DT, VEC, PASS, RUNS, WARPS>;
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
    cfg.attrs = attr; cfg.numAttrs = pdl_enabled("linear_fp8") ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, map[0], map[1], D);
}

template <int DT, bool VEC>
cudaError_t choose(const Fp8Linear &P, cudaStream_t st)
{
    if (ceil_div(P.M, GROUP) > 2 * device_sm_count()) return run<DT, VEC, 5, false, 8>(P, st);
    // up to two groups a CTA: a block is mostly waits, for 16 warps to overlap
    return P.N % FP8_BLOCK == 0 ? run<DT, VEC, 2, true, 16>(P, st) : run<DT, VEC, 2, false, 16>(P, st);
}

}  // namespace

cudaError_t launch_linear_fp8_decode(const Fp8Linear &P, cudaStream_t st)
{
    const bool vec = P.N % 8 == 0;
    switch (P.x_dtype) {
    case VPTQ_DTYPE_E4M3: return choose<VPTQ_DTYPE_E4M3, true>(P, st);
    case VPTQ_DTYPE_BF16: return vec ? choose<VPTQ_DTYPE_BF16, true>(P, st) : choose<VPTQ_DTYPE_BF16, false>(P, st);
    default: return vec ? choose<VPTQ_DTYPE_FP16, true>(P, st) : choose<VPTQ_DTYPE_FP16, false>(P, st);
    }
}

}  // namespace vptq
