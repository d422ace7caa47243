// out = x W^T for more than 8 tokens over an e4m3 weight with 128 x 128 block scales, on the tensor cores.
//
// D[token][feature] per block of 128 columns is one group of four tcgen05.mma (kind::f8f6f4, 128 tokens x TN features x 32 columns
// each) into a TMEM buffer of its own; the block's two scales differ from the next block's, so the sum over blocks is formed in
// registers: acc += D * (x_scale[token][block] * w_scale[feature block][block]).  A TMEM lane is a token: its scale is one register of
// the lane, the weight's is the same for 128 columns, and the update is one packed fma per two values.
//
// Warps by role: 0 loads (TMA, 128-byte swizzle, zeros beyond the matrices' edges), 1 issues the MMAs, 2 and 3 bring the blocks' scales to
// shared memory (read by the lanes that use them they lie a row apart, 32 cache lines to a load), 4..11 read the buffers and hold the
// sums (two warps per lane quarter, half a tile's features each).  Two TMEM buffers: one fills while the other is read.
// CTAs are persistent over tiles, tokens fastest, so that those that run together share weight tiles in L2.
// Few tiles: SPLIT CTAs of a cluster share a tile's columns, leave their sums in shared memory, and each adds up its share of the
// tile's rows in rank order: one launch, no scratch, and a result that does not depend on timing.
// Bound by the two L2-side and issue-side halves of a block, operand tiles at 50 to 55 bytes a clock and SM and the sums' fmas, which overlap only
// partly: 8192 x 28672 at 2048 tokens 475 us sustained, 2030 TFLOP/s; 8192 x 8192 at 2048 121 us (103 without the loads, 106 without the fmas).
// Few tokens: HBM (28672 x 8192 at 16 tokens 46 us, 5.1 TB/s).
// Every wait is bounded.  A warp whose wait gives up stops: it loads, multiplies or hands on nothing more, so that the waits that depend
// on it run out too and no sum is made of what has not arrived.  The results of warps that gave up are NaN, and the workspace's status word is set.
#include "fp8.cuh"
#include "fp8_tcgen05.cuh"
#include "tcgen05_pair.cuh"

namespace vptq {

namespace {

using namespace tc;

constexpr int TM = 128;                                   // tokens of a tile
constexpr int SCALE_WARP0 = 2, SCALE_WARPS = 2, ACC_WARP0 = 4, ACC_WARPS = 8;
constexpr int THREADS = 32 * (ACC_WARP0 + ACC_WARPS);
// Registers: 12 warps of 168 at launch; the first four give some up, the others hold up to 128 sums and 32 loaded values a lane
// (4 x 104 + 8 x 200 = 12 x 168).  A loop with spills is lost: the stages leave L1 next to nothing, so a reload is a trip to L2.
constexpr int FEW_REGS = 104, ACC_REGS = 200;
constexpr int X_BYTES = TM * FP8_BLOCK;                   // a stage's activations
constexpr int STAGING = 2048;                             // per accumulating warp: 32 rows x 16 columns on their way out
constexpr int SMEM_MAX = 232448 - 1024;                  // (the static part takes a multiple of the dynamic part's alignment)
constexpr int BARRIERS = 256;
constexpr int SCALE_KBS = 16;                             // blocks of columns whose scales are brought in together
constexpr int SCALE_BYTES = SCALE_KBS * (TM + 4) * 4;     // [SCALE_KBS][TM] of the tokens, [SCALE_KBS][4] of the features' 128-row blocks
constexpr int FIXED_BYTES = ACC_WARPS * STAGING + 2 * SCALE_BYTES + BARRIERS;

// a CTA's part of a stage: its tokens, and the tile's features or (pairs) half of them
template <int TN, int PAIR> constexpr int stage_bytes() { return X_BYTES + TN / PAIR * FP8_BLOCK; }
template <int TN, int PAIR> constexpr int stages()
{
    const int n = (SMEM_MAX - FIXED_BYTES) / stage_bytes<TN, PAIR>();
    return n < 8 ? n : 8;
}
template <int TN, int PAIR> constexpr int smem_bytes() { return stages<TN, PAIR>() * stage_bytes<TN, PAIR>() + FIXED_BYTES; }
struct Params {
    int M, B, kbs;
    int tiles_t, tiles;
    const float *x_scale, *w_scale;
    void *out;
    int out_dtype;
    int tma_out;           // rows of `out` are 16-byte aligned: stored by TMA
    int *status;
    unsigned long long wait_limit;
};

template <int PAIR>
__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    if constexpr (PAIR == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

__device__ __forceinline__ void fma2(uint64_t &acc, uint64_t a, uint64_t b) { asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc) : "l"(a), "l"(b)); }

// What the accumulating warps need of a CTA.
struct Sums {
    uint32_t tmem, staging;
    uint8_t *staging_p, *sm;
    uint32_t lost_at;                      // shared memory: not 0 when a wait of the CTA's other warps gave up
    const float *scales;                   // two buffers of SCALE_BYTES
    uint32_t acc_full, acc_empty, scale_full, scale_empty;      // barriers, the first of two each
    int first, step, kb0, kb1;             // tiles and columns
    int t_rank;                            // pairs: this CTA's tokens of a tile start at t_rank * TM
};

// where token `row`'s scale lies in a buffer's line of TM: lines are written by 16 lanes at a time, one line each, and read along
__device__ __forceinline__ int scale_slot(int line, int row) { return line * TM + (row ^ (2 * line)); }

// NaN to `rows` x `cols` values of the result; thread `i` of n
__device__ __forceinline__ void store_nan(const Params &P, int row, int rows, int col, int cols, int i, int n)
{
    for (int r = 0; r < rows; r++)
        for (int c = i; c < cols; c += n) store_out(P.out, (long long)(row + r) * P.M + col + c, __int_as_float(0x7FFFFFFF), P.out_dtype);
}

// Sums of half a tile's features, from c_first on, of the 32 tokens of lane quarter q.
template <int TN, int SPLIT, int PAIR>
__device__ __forceinline__ void accumulate(const CUtensorMap &map_out, const Params &P, const Sums &S, int c_first, int q, int lane, uint32_t &gave_up)
{
    constexpr int COUNT = TN / 2, CHUNKS = COUNT / 16;
    uint32_t it = 0, group = 0, pieces = 0;
    for (int tile = S.first; tile < P.tiles; tile += S.step) {
        const int t0 = (tile % P.tiles_t * PAIR + S.t_rank) * TM, n0 = tile / P.tiles_t * TN;
        // 128-row blocks of the weight that the features lie in: one, or two from feature `second` on
        const int block = (n0 + c_first) / FP8_BLOCK - n0 / FP8_BLOCK, second = FP8_BLOCK - (n0 + c_first) % FP8_BLOCK;
        uint64_t acc[COUNT / 2];
#pragma unroll
        for (int i = 0; i < COUNT / 2; i++) acc[i] = 0;
#pragma unroll 1
        for (int kb = S.kb0; kb < S.kb1; kb++, it++) {
            const uint32_t buf = it & 1, taddr = S.tmem + buf * 256;
            const int line = (kb - S.kb0) % SCALE_KBS;
            if (line == 0) mbar_wait_or_flag(S.scale_full + 8 * (group & 1), (group >> 1) & 1, S.lost_at, gave_up);
            const float *scales = S.scales + (group & 1) * (SCALE_BYTES / 4), *ws = scales + SCALE_KBS * TM + 4 * line + block;
            const float xs = scales[scale_slot(line, 32 * q + lane)], s0 = xs * ws[0], s1 = xs * ws[1];
            if (line == SCALE_KBS - 1 || kb == S.kb1 - 1) {
                __syncwarp();
                if (lane == 0 && !gave_up) mbar_arrive(S.scale_empty + 8 * (group & 1));
                group++;
            }
            mbar_wait_or_flag(S.acc_full + 8 * buf, (it >> 1) & 1, S.lost_at, gave_up);
            tc_fence_after();
            uint32_t d[2][16];
            tmem_start16(taddr, d[0]);
#pragma unroll
            for (int j = 0; j < CHUNKS; j++) {
                tmem_wait16(d[j & 1]);
                if (j + 1 < CHUNKS) tmem_start16(taddr + 16 * (j + 1), d[(j + 1) & 1]);
                else {
                    // everything read: the buffer is the MMA warp's again
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0 && !gave_up) {
                        if (PAIR == 2) arrive_in_cluster(S.acc_empty + 8 * buf);
                        else mbar_arrive(S.acc_empty + 8 * buf);
                    }
                }
                const float sf = 16 * j < second ? s0 : s1;
                const uint64_t ss = pack2(__float_as_uint(sf), __float_as_uint(sf));
#pragma unroll
                for (int i = 0; i < 8; i++) fma2(acc[8 * j + i], pack2(d[j & 1][2 * i], d[j & 1][2 * i + 1]), ss);
            }
        }
        if constexpr (SPLIT > 1) {
            // the tile's sums over this CTA's columns: [128][TN] FP32 where the stages were (the last MMAs, which this warp has seen
            // end, were the last to read those); 16-byte pieces of a row exchanged so that the lanes of a quarter warp write different banks
#pragma unroll
            for (int j = 0; j < COUNT / 4; j++) {
                const float2 a = unpack2(acc[2 * j]), b = unpack2(acc[2 * j + 1]);
                const int row = 32 * q + lane, piece = (c_first / 4 + j) ^ (lane & 7);
                *reinterpret_cast<float4 *>(S.sm + (row * TN + 4 * piece) * 4) = make_float4(a.x, a.y, b.x, b.y);
            }
        } else {
            // 16 features at a time through the warp's staging rows (32 or 64 bytes, swizzled as the store's map says)
            const bool wide = P.out_dtype == VPTQ_DTYPE_FP32;
#pragma unroll
            for (int j = 0; j < CHUNKS; j++) {
                // (16-bit pieces take turns at two halves of the staging; every piece is a group of its own, stored or not)
                const uint32_t at = wide ? 0u : (pieces++ & 1) * (STAGING / 2);
                if (P.tma_out && lane == 0) {
                    if (wide) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    else asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                }
                __syncwarp();
                if (wide) {
#pragma unroll
                    for (int c = 0; c < 4; c++) {
                        const float2 a = unpack2(acc[8 * j + 2 * c]), b = unpack2(acc[8 * j + 2 * c + 1]);
                        *reinterpret_cast<float4 *>(S.staging_p + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4)) = make_float4(a.x, a.y, b.x, b.y);
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < 2; c++) {
                        uint32_t h[4];
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            const float2 a = unpack2(acc[8 * j + 4 * c + i]);
                            h[i] = pair16(a.x, a.y, P.out_dtype);
                        }
                        *reinterpret_cast<uint4 *>(S.staging_p + at + lane * 32 + ((c ^ ((lane >> 2) & 1)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
                    }
                }
                const int col = n0 + c_first + 16 * j;
                if (P.tma_out) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        if (col < P.M && t0 + 32 * q < P.B) tma_store(&map_out, S.staging + at, col, t0 + 32 * q);
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                } else {
                    __syncwarp();
                    const int c = lane & 15;
                    for (int r = lane >> 4; r < 32 && t0 + 32 * q + r < P.B; r += 2) {
                        if (col + c >= P.M) break;
                        const long long o = (long long)(t0 + 32 * q + r) * P.M + col + c;
                        if (wide) reinterpret_cast<float *>(P.out)[o] = *reinterpret_cast<const float *>(S.staging_p + r * 64 + (((c >> 2) ^ ((r >> 1) & 3)) << 4) + (c & 3) * 4);
                        else reinterpret_cast<uint16_t *>(P.out)[o] = *reinterpret_cast<const uint16_t *>(S.staging_p + at + r * 32 + (((c >> 3) ^ ((r >> 2) & 1)) << 4) + (c & 7) * 2);
                    }
                    __syncwarp();
                }
            }
            // A lane that gave up went on without handing anything on; the warp's sums are no good whichever lane it was.  (NaN is written over them:
            // put into the registers of the sums, or into the values on their way out, it cost 20 us of 8192 x 28672 at 2048 tokens.)
            if (__any_sync(0xffffffffu, load_word(S.lost_at) != 0)) {
                if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
                __syncwarp();
                const int rows = min(32, P.B - t0 - 32 * q), cols = min(COUNT, P.M - n0 - c_first);
                store_nan(P, t0 + 32 * q, rows, n0 + c_first, cols, lane, 32);
            }
        }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

template <int TN, int SPLIT, int PAIR>
__global__ void __launch_bounds__(THREADS, 1)
linear_fp8_tcgen05_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_out,
                          const __grid_constant__ Params P)
{
    constexpr int ST = stages<TN, PAIR>(), SB = stage_bytes<TN, PAIR>();
    extern __shared__ __align__(1024) uint8_t sm[];
    __shared__ uint32_t tmem_slot, lost;                  // lost: a wait of this CTA gave up (of a pair: of either)
    const uint32_t base = smem_addr(sm), staging0 = base + ST * SB, bars = staging0 + FIXED_BYTES - BARRIERS;
    float *scales = reinterpret_cast<float *>(sm + ST * SB + ACC_WARPS * STAGING);
    auto bar_full = [&](int s) { return bars + 8u * s; };
    auto bar_empty = [&](int s) { return bars + 8u * (ST + s); };
    auto bar_acc_full = [&](int b) { return bars + 8u * (2 * ST + b); };
    auto bar_acc_empty = [&](int b) { return bars + 8u * (2 * ST + 2 + b); };
    auto bar_scale_full = [&](int b) { return bars + 8u * (2 * ST + 4 + b); };
    auto bar_scale_empty = [&](int b) { return bars + 8u * (2 * ST + 6 + b); };
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        lost = 0;
        for (int s = 0; s < ST; s++) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 1); }
        for (int b = 0; b < 2; b++) { mbar_init(bar_acc_full(b), 1); mbar_init(bar_acc_empty(b), PAIR * ACC_WARPS); mbar_init(bar_scale_full(b), SCALE_WARPS); mbar_init(bar_scale_empty(b), ACC_WARPS); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        tmem_alloc_all<PAIR>(smem_addr(&tmem_slot));
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR == 2) cluster_sync();              // the other CTA's barriers are ready, and its half of TMEM
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    pdl_launch_dependents();

    // this CTA's tiles and columns
    const int rank = SPLIT * PAIR > 1 ? (int)cluster_rank() : 0, t_rank = PAIR > 1 ? rank : 0;
    const int first = (int)blockIdx.x / (SPLIT * PAIR), step = SPLIT > 1 ? P.tiles : (int)gridDim.x / PAIR;
    const int kb0 = SPLIT > 1 ? (int)((long long)P.kbs * rank / SPLIT) : 0, kb1 = SPLIT > 1 ? (int)((long long)P.kbs * (rank + 1) / SPLIT) : P.kbs;
    const uint32_t lost_at = smem_addr(&lost);
    uint32_t gave_up = 0;
    auto report = [&]() {                                 // (at the end of a role: to both CTAs of a pair, which leave together)
        if (__any_sync(0xffffffffu, gave_up != 0) && lane == 0) {
            if (PAIR == 2) { store_peer_word(lost_at, 0, 1); store_peer_word(lost_at, 1, 1); }
            else *reinterpret_cast<volatile uint32_t *>(&lost) = 1;
        }
        __syncwarp();
    };

    if (warp < ACC_WARP0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(FEW_REGS));
        if (warp == 0) {
            // ---- loads: this CTA's tokens, and its part of the tile's features; the bytes of a pair count on rank 0's barrier ----
            uint32_t it = 0;
            const uint32_t full0 = PAIR > 1 ? address_in(bar_full(0), 0) : bar_full(0);
            const int n_part = t_rank * (TN / PAIR);
            pdl_wait();                                                        // (weight and activations may be the preceding kernel's)
            for (int tile = first; tile < P.tiles; tile += step) {
                const int t0 = (tile % P.tiles_t * PAIR + t_rank) * TM, n0 = tile / P.tiles_t * TN + n_part;
                for (int kb = kb0; kb < kb1; kb++, it++) {
                    const uint32_t s = it % ST;
                    mbar_wait_or_flag(bar_empty(s), ((it / ST) & 1) ^ 1u, lost_at, gave_up);
                    if (elect_one() && !gave_up) {
                        if (t_rank == 0) mbar_expect_tx(bar_full(s), PAIR * SB);
                        tma_load<PAIR>(base + s * SB + X_BYTES, &map_w, kb * FP8_BLOCK, n0, full0 + 8 * s);
                        tma_load<PAIR>(base + s * SB, &map_x, kb * FP8_BLOCK, t0, full0 + 8 * s);
                    }
                    __syncwarp();
                }
            }
        } else if (warp == 1) {
            // ---- MMAs: e4m3 x e4m3 -> FP32, both K-major; of a pair, rank 0's over the memory of both ----
            constexpr uint32_t IDESC = (1u << 4) | ((uint32_t)(TN >> 3) << 17) | ((uint32_t)(PAIR * TM >> 4) << 24);
            const uint64_t a0 = make_smem_desc(base, 16, 1024, LAYOUT_SW128), b0 = make_smem_desc(base + X_BYTES, 16, 1024, LAYOUT_SW128);
            uint32_t it = 0;
            pdl_wait();                                                        // (a wait's time does not begin before the preceding kernel has ended)
            for (int tile = first; tile < P.tiles && t_rank == 0; tile += step)
                for (int kb = kb0; kb < kb1; kb++, it++) {
                    const uint32_t s = it % ST, buf = it & 1;
                    mbar_wait_flagged(bar_full(s), (it / ST) & 1, P.wait_limit, lost_at, gave_up);
                    mbar_wait_or_flag(bar_acc_empty(buf), ((it >> 1) & 1) ^ 1u, lost_at, gave_up);
                    tc_fence_after();
                    if (elect_one() && !gave_up) {
                        const uint64_t at = (uint64_t)((s * SB) >> 4);
#pragma unroll
                        for (int k = 0; k < FP8_BLOCK / 32; k++) mma_f8<PAIR>(tmem + buf * 256, a0 + at + 2 * k, b0 + at + 2 * k, IDESC, k > 0);
                        commit<PAIR>(bar_acc_full(buf));
                        commit<PAIR>(bar_empty(s));
                    }
                    __syncwarp();
                }
        } else {
            // ---- scales: 16 blocks of columns at a time, along the rows they are stored in; the sums read them across ----
            pdl_wait();                                                        // the activations' may be the preceding kernel's
            const int line = lane & 15, odd = lane >> 4, part = warp - SCALE_WARP0;
            uint32_t group = 0;
            for (int tile = first; tile < P.tiles; tile += step) {
                const int t0 = (tile % P.tiles_t * PAIR + t_rank) * TM, n0 = tile / P.tiles_t * TN, rows = min(TM, P.B - t0);
                for (int kb = kb0; kb < kb1; kb += SCALE_KBS, group++) {
                    float *buf = scales + (group & 1) * (SCALE_BYTES / 4);
                    mbar_wait_or_flag(bar_scale_empty(group & 1), ((group >> 1) & 1) ^ 1u, lost_at, gave_up);
                    // (Scales of a wait that gave up go into a buffer that may be in use: whoever reads them finds `lost` at the tile's end.  A way
                    // out of the loop here, or conditional stores, would keep the loads from being under way early and together: 8192 x 28672 at
                    // 2048 tokens 485 us, 522 and 590.)
                    const bool in = kb + line < kb1;
                    const float *src = P.x_scale + (long long)t0 * P.kbs + kb + line;
#pragma unroll 8
                    for (int row = 2 * part + odd; row < TM; row += 2 * SCALE_WARPS)
                        buf[scale_slot(line, row)] = in && row < rows ? __ldg(src + (long long)row * P.kbs) : 0.f;
                    if (part == 0)
#pragma unroll
                        for (int j = 0; j < 4; j += 2) {
                            const int block = min(n0 / FP8_BLOCK + j + odd, (P.M - 1) / FP8_BLOCK);
                            buf[SCALE_KBS * TM + 4 * line + j + odd] = in ? __ldg(P.w_scale + (long long)block * P.kbs + kb + line) : 0.f;
                        }
                    __syncwarp();
                    if (lane == 0 && !gave_up) mbar_arrive(bar_scale_full(group & 1));
                }
            }
        }
        report();
        if constexpr (SPLIT > 1) {
            cluster_sync();
            cluster_sync();
        }
    } else {
        // ---- sums ----
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(ACC_REGS));
        const int w = warp - ACC_WARP0, q = warp & 3, share = w >> 2;          // TMEM lane quarter this warp may read, its part of the features
        pdl_wait();                                                            // (the result, and the status word, may be the preceding kernel's)
        if (blockIdx.x == 0 && threadIdx.x == 32 * ACC_WARP0) *P.status = 0;
        const Sums S = {tmem + ((uint32_t)(32 * q) << 16) + share * (TN / 2), staging0 + w * STAGING, sm + ST * SB + w * STAGING, sm, lost_at, scales,
                        bar_acc_full(0), PAIR > 1 ? address_in(bar_acc_empty(0), 0) : bar_acc_empty(0), bar_scale_full(0), bar_scale_empty(0), first, step, kb0, kb1, t_rank};
        accumulate<TN, SPLIT, PAIR>(map_out, P, S, share * (TN / 2), q, lane, gave_up);
        report();
        if constexpr (SPLIT > 1) {
            cluster_sync();
            const uint32_t peer_lost = lane < SPLIT ? load_peer_word(lost_at, (uint32_t)lane) : 0u;       // (looked at below: no wait for it here)
            // rows of the tile that are tokens, dealt out over the ranks; four features a thread, the ranks' sums added in order
            const int t0 = first % P.tiles_t * TM, n0 = first / P.tiles_t * TN;
            const int rows = min(TM, P.B - t0), r0 = rows * rank / SPLIT, r1 = rows * (rank + 1) / SPLIT;
            constexpr int PIECES = TN / 4;
            for (int i = threadIdx.x - 32 * ACC_WARP0; i < (r1 - r0) * PIECES; i += 32 * ACC_WARPS) {
                const int row = r0 + i / PIECES, p = i % PIECES, col = n0 + 4 * p;
                const uint32_t at = base + (uint32_t)(row * TN + 4 * (p ^ (row & 7))) * 4u;
                float4 v[SPLIT];
#pragma unroll
                for (int r = 0; r < SPLIT; r++) v[r] = load_peer(at, (uint32_t)r);
#pragma unroll
                for (int r = 1; r < SPLIT; r++) { v[0].x += v[r].x; v[0].y += v[r].y; v[0].z += v[r].z; v[0].w += v[r].w; }
                const long long o = (long long)(t0 + row) * P.M + col;
                if (P.tma_out && col + 4 <= P.M) {                                 // rows of 16-byte multiples: a thread's four values are aligned
                    if (P.out_dtype == VPTQ_DTYPE_FP32) *reinterpret_cast<float4 *>(reinterpret_cast<float *>(P.out) + o) = v[0];
                    else *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(P.out) + o) = make_uint2(pair16(v[0].x, v[0].y, P.out_dtype), pair16(v[0].z, v[0].w, P.out_dtype));
                } else {
                    const float e[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
                    for (int k = 0; k < 4; k++)
                        if (col + k < P.M) store_out(P.out, o + k, e[k], P.out_dtype);
                }
            }
            __syncwarp();
            if (__any_sync(0xffffffffu, peer_lost != 0)) {                     // (the same for every warp)
                asm volatile("bar.sync 1, %0;" ::"n"(32 * ACC_WARPS) : "memory");
                store_nan(P, t0 + r0, r1 - r0, n0, min(TN, P.M - n0), threadIdx.x - 32 * ACC_WARP0, 32 * ACC_WARPS);
            }
            __syncwarp();
            cluster_sync();                                                    // a peer may still read this CTA's sums
        }
    }
    // (what the warps run together from here on has to do with the registers that the first four kept)
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR == 2) cluster_sync();              // neither CTA leaves while the other's MMAs, copies or arrivals need it
    if (*reinterpret_cast<volatile uint32_t *>(&lost)) {
        let_copies_land();
        if (threadIdx.x == 0) atomicExch(P.status, VPTQ_E_TIMEOUT);            // (long after the word was cleared)
        __syncthreads();
        if constexpr (PAIR == 2) cluster_sync();
    }
    if (warp == 1) {
        tc_fence_after();
        tmem_free_all<PAIR>(tmem);
    }
}

// ---- host side ----------------------------------------------------------------------------------------

template <int TN, int SPLIT, int PAIR>
cudaError_t run(const Fp8Linear &L, const Params &P0, cudaStream_t st)
{
    Params P = P0;
    const long long pitch = fp8_row_bytes(L.N), out_bytes = L.out_dtype == VPTQ_DTYPE_FP32 ? 4 : 2;
    CUtensorMap map_x, map_w, map_out;
    if (!encode_tensor_map(&map_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, L.x, pitch, L.B, pitch, 0, 0, FP8_BLOCK, TM, 1, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !encode_tensor_map(&map_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, L.w, pitch, L.M, pitch, 0, 0, FP8_BLOCK, TN / PAIR, 1, CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorNotSupported;
    map_out = map_x;                                      // (not read unless tma_out)
    P.tma_out = L.M * out_bytes % 16 == 0 ? 1 : 0;
    if (P.tma_out &&
        !encode_tensor_map(&map_out, out_bytes == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, L.out, L.M, L.B, L.M * out_bytes, 0, 0, 16, 32, 1,
                           out_bytes == 4 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B))
        return cudaErrorNotSupported;
    P.tiles_t = ceil_div(L.B, PAIR * TM);
    P.tiles = P.tiles_t * ceil_div(L.M, TN);
    auto kern = linear_fp8_tcgen05_kernel<TN, SPLIT, PAIR>;
    constexpr int SMEM = smem_bytes<TN, PAIR>(), CLUSTER = SPLIT * PAIR;
    const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void *>(kern), SMEM);
    if (e != cudaSuccess) return e;
    int resident = device_sm_count();                     // clusters that work at a time
    if (PAIR > 1) {
        resident = max_resident_clusters(reinterpret_cast<const void *>(kern), CLUSTER, THREADS, SMEM);
        if (resident < 1) return cudaErrorNotSupported;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(CLUSTER * (SPLIT > 1 || P.tiles < resident ? P.tiles : resident)));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (CLUSTER > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = CLUSTER; attr[n].val.clusterDim.y = 1; attr[n].val.clusterDim.z = 1;
        n++;
    }
    if (pdl_enabled("linear_fp8")) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        n++;
    }
    cfg.attrs = attr; cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kern, map_x, map_w, map_out, P);
}

// split tiles that work at a time: clusters of 8 do not fill the device (an SM partition holds two)
int resident_splits(int tn, int split)
{
    const void *kern = tn == 64 ? (split == 2 ? (const void *)linear_fp8_tcgen05_kernel<64, 2, 1> : split == 4 ? (const void *)linear_fp8_tcgen05_kernel<64, 4, 1>
                                                                                                               : (const void *)linear_fp8_tcgen05_kernel<64, 8, 1>)
                                : (split == 2 ? (const void *)linear_fp8_tcgen05_kernel<128, 2, 1> : split == 4 ? (const void *)linear_fp8_tcgen05_kernel<128, 4, 1>
                                                                                                                 : (const void *)linear_fp8_tcgen05_kernel<128, 8, 1>);
    return max_resident_clusters(kern, split, THREADS, tn == 64 ? smem_bytes<64, 1>() : smem_bytes<128, 1>());
}

struct Choice { int tn, split, pair; };

// Tile width, split and pairs by estimated time.  Measured at 8192 x 8192 and 2048 tokens: ns per block of 128 columns of a tile, every SM
// at work.  Wide tiles bring fewer bytes in from L2 per product, pairs, which bring half of a tile's features to each of two SMs, fewer
// still, but every block of theirs waits for both; 224 alone (491) and 192 (442) and 256 (502) in pairs are never the fastest.  A tile
// ends with about 0.9 us for its results, a split one with 1.5 for the meeting.
Choice choose(int M, int B, int kbs)
{
    constexpr int WIDTHS = 6;
    const int widths[WIDTHS] = {256, 224, 192, 160, 128, 64}, splits[4] = {1, 2, 4, 8};
    const double block_ns[2][WIDTHS] = {{491, 0, 441, 401, 360, 287}, {0, 469, 0, 367, 313, 0}};      // 0: there is no such kernel
    const int sms = device_sm_count();
    Choice best = {256, 1, 1};
    double best_time = 1e300;
    for (int pair = 1; pair <= 2; pair++)
        for (int i = 0; i < WIDTHS; i++)
            for (int j = 0; j < 4; j++) {
                const int tn = widths[i], split = splits[j];
                if (block_ns[pair - 1][i] == 0 || (pair > 1 && B <= TM)) continue;
                if (split > 1 && (tn > 128 || kbs < 2 * split || pair > 1)) continue;
                const long long tiles = (long long)ceil_div(B, pair * TM) * ceil_div(M, tn);
                if (split > 1 && tiles > resident_splits(tn, split)) continue;
                const long long waves = split > 1 ? 1 : (tiles + sms / pair - 1) / (sms / pair);
                const double time = waves * (ceil_div(kbs, split) * block_ns[pair - 1][i] + (split > 1 ? 1500 : 900));
                if (time < best_time) { best_time = time; best = {tn, split, pair}; }
            }
    return best;
}

}  // namespace

cudaError_t launch_linear_fp8_tcgen05(const Fp8Linear &L, int *status, cudaStream_t st)
{
    Params P;
    P.M = L.M; P.B = L.B; P.kbs = ceil_div(L.N, FP8_BLOCK);
    P.x_scale = L.x_scale; P.w_scale = L.w_scale; P.out = L.out; P.out_dtype = L.out_dtype; P.status = status;
    P.wait_limit = wait_limit();
    P.tiles_t = P.tiles = P.tma_out = 0;
    const Choice c = choose(L.M, L.B, P.kbs);
    if (c.pair == 2) switch (c.tn) {
        case 224: return run<224, 1, 2>(L, P, st);
        case 160: return run<160, 1, 2>(L, P, st);
        default: return run<128, 1, 2>(L, P, st);
        }
    switch (c.tn * 10 + c.split) {
    case 2561: return run<256, 1, 1>(L, P, st);
    case 1921: return run<192, 1, 1>(L, P, st);
    case 1601: return run<160, 1, 1>(L, P, st);
    case 1281: return run<128, 1, 1>(L, P, st);
    case 1282: return run<128, 2, 1>(L, P, st);
    case 1284: return run<128, 4, 1>(L, P, st);
    case 1288: return run<128, 8, 1>(L, P, st);
    case 641: return run<64, 1, 1>(L, P, st);
    case 642: return run<64, 2, 1>(L, P, st);
    case 644: return run<64, 4, 1>(L, P, st);
    default: return run<64, 8, 1>(L, P, st);
    }
}

}  // namespace vptq
