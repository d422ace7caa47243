// out = x W^T over e2m1 operands with a power of two for every 32 columns of a row, on the tensor cores.
//
// D[token][feature] is a sum of tcgen05.mma (kind::mxf4, 128 tokens x TN features x 64 columns each) which multiply every block's products
// with its two scales themselves, so that a tile's whole sum stays in TMEM.  The scales go there too, as the instruction wants them: a tile
// of 128 rows x 4 blocks, in the order in which it lies in memory (fp4.cuh), is copied to four columns by one tcgen05.cp, which the MMAs
// issued behind it wait for by themselves.
//
// Warps by role: 0 loads (TMA: operands with 128-byte swizzle, zeros beyond the matrices' edges; scale tiles as they are), 1 copies scales
// and issues the MMAs, 4..11 read the sums (two warps per lane quarter, half a tile's features each) into registers at once, so that the next
// tile's MMAs begin while they convert and store.
// CTAs are persistent over tiles, tokens fastest, so that those that run together share weight tiles in L2.
// Few tiles: SPLIT CTAs of a cluster share a tile's columns, leave their sums in shared memory, and each adds up its share of the
// tile's rows in rank order: one launch, no scratch, and a result that does not depend on timing.
// Every wait is bounded.  A warp whose wait gives up stops: it loads, multiplies or hands on nothing more, so that the waits that depend
// on it run out too and no sum is made of what has not arrived.  The results of a CTA with a wait that gave up are NaN, and the workspace's status word is set.
#include <math.h>

#include "fp4.cuh"
#include "fp4_tcgen05.cuh"
#include "tcgen05_pair.cuh"

namespace vptq {

namespace {

using namespace tc;

constexpr int TM = 128;                                   // tokens of a tile
constexpr int KB = 256, KB_BYTES = KB / 2;                // columns of a stage: a swizzled row of 128 bytes
constexpr int STEPS = KB / 64, CHUNKS = KB / FP4_TILE_COLS;            // MMAs, and scale tiles of 128 rows, along a stage
constexpr int ACC_WARP0 = 4, ACC_WARPS = 8;
constexpr int THREADS = 32 * (ACC_WARP0 + ACC_WARPS);
// Registers: 12 warps of 168 at launch; the first four give some up, the others hold up to 128 sums a lane (4 x 104 + 8 x 200 = 12 x 168).
constexpr int FEW_REGS = 104, ACC_REGS = 200;
constexpr int SCALES = CHUNKS * FP4_TILE_BYTES;           // of 128 rows, along a stage
constexpr int STAGING = 4096;                             // per accumulating warp: 32 rows of 128 bytes on their way out
constexpr int SMEM_MAX = 232448 - 1024;                  // (the static part takes a multiple of the dynamic part's alignment)
constexpr int BARRIERS = 256;
constexpr int FIXED_BYTES = ACC_WARPS * STAGING + BARRIERS;

// 128-row tiles of the weight's scales that a tile's features lie in
template <int TN> constexpr int row_tiles() { return TN > 128 ? 2 : 1; }
// a CTA's part of a stage beside its tokens: the tile's features or (pairs) half of them, scales of 128 tokens and of all of the tile's features
template <int TN, int PAIR> constexpr int weight_bytes() { return TN / PAIR * KB_BYTES + (1 + row_tiles<TN>()) * SCALES; }
// stages that fit, at most MAX_STAGES.  Few tokens take less of a stage: an MMA reads 128 rows all the same, into what follows (behind the last stage that
// is the staging), for sums that nobody reads.
constexpr int MAX_STAGES = 12;
template <int TN, int PAIR> constexpr int stages(int x_bytes)
{
    const int n = (SMEM_MAX - FIXED_BYTES) / (x_bytes + weight_bytes<TN, PAIR>());
    return n < MAX_STAGES ? n : MAX_STAGES;
}
// TMEM columns: one buffer of sums, or two; behind them two of scales, taken in turn by the stages
template <int TN> constexpr int buffers() { return TN <= 128 ? 2 : 1; }
// features that an accumulating warp takes: at least a piece of 128 bytes of 16-bit results (a tile of 64: four of the warps take all)
template <int TN> constexpr int count() { return TN >= 128 ? TN / 2 : TN; }
constexpr int SCALE_COLS = 32;

struct Params {
    int M, B, kbs, last_steps;
    int col_tiles, row_tiles;              // scale tiles along a row of 128-row tiles, and of those rows the weight's
    const uint8_t *x_scale, *w_scale;
    int tiles_t, tiles;
    int x_bytes, stages;                   // of a CTA's part of a stage: activations; stages of the ring
    void *out;
    int out_dtype;
    int tma_out;           // rows of `out` are 16-byte aligned: stored by TMA
    int *status;
    int weight_early;      // all that came before the preceding kernel of the stream has ended, and that one does not write the weight
    unsigned long long wait_limit;
};

template <int PAIR>
__device__ __forceinline__ void mma_fp4(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t a_scale, uint32_t b_scale, uint32_t accumulate)
{
    if constexpr (PAIR == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(a_scale), "r"(b_scale), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(a_scale), "r"(b_scale), "r"(accumulate) : "memory");
}
// a scale tile (32 rows of 16 bytes in shared memory) to four TMEM columns, for all four lane quarters; of a pair, in both CTAs
template <int PAIR>
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc)
{
    if constexpr (PAIR == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}

// NaN to `rows` x `cols` values of the result; thread `i` of n
__device__ __forceinline__ void store_nan(const Params &P, int row, int rows, int col, int cols, int i, int n)
{
    for (int r = 0; r < rows; r++)
        for (int c = i; c < cols; c += n) store_out(P.out, (long long)(row + r) * P.M + col + c, __int_as_float(0x7FFFFFFF), P.out_dtype);
}

// What the accumulating warps need of a CTA.
struct Sums {
    uint32_t tmem, staging;
    uint8_t *staging_p, *sm;
    uint32_t lost_at;                      // shared memory: not 0 when a wait of the CTA's other warps gave up
    uint32_t acc_full, acc_empty;          // barriers, the first of buffers<TN>() each
    int first, step;                       // tiles
    int t_rank;                            // pairs: this CTA's tokens of a tile start at t_rank * TM
};

// 128 bytes of features from `col` on of 32 tokens from `row` on; `chunk` gives a lane's 16 bytes at place c of its row
template <bool WIDE, typename Chunk>
__device__ __forceinline__ void store_piece(const CUtensorMap &map_out, const Params &P, const Sums &S, int lane, int row, int col, Chunk chunk)
{
    constexpr int SIZE = WIDE ? 4 : 2;
    if (P.tma_out && lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 8; c++) *reinterpret_cast<uint4 *>(S.staging_p + lane * 128 + ((c ^ (lane & 7)) << 4)) = chunk(c);
    if (P.tma_out) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            if (col < P.M) tma_store(&map_out, S.staging, col, row);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
    } else {
        __syncwarp();
        // a lane's four bytes of eight rows at a time; two 16-bit results go out apart where M is odd and every other row begins between words.  (Row by row,
        // value by value: 5001 x 700 at 2000 tokens 35 us instead of 15)
        const int c = col + lane * (4 / SIZE), rows = min(32, P.B - row);
        uint8_t *o = reinterpret_cast<uint8_t *>(P.out) + ((long long)row * P.M + c) * SIZE;
        const long long step = (long long)P.M * SIZE;
        const bool in = c < P.M, both = WIDE || c + 1 < P.M, apart = !WIDE && ((P.M & 1) || !both);
        const uint8_t *at = S.staging_p + (lane & 3) * 4;
#pragma unroll 1
        for (int r0 = 0; r0 < rows; r0 += 8) {
            uint32_t v[8];
#pragma unroll
            for (int r = 0; r < 8; r++) v[r] = *reinterpret_cast<const uint32_t *>(at + (r0 + r) * 128 + ((lane >> 2 ^ r) << 4));
            if (apart) {
#pragma unroll
                for (int r = 0; r < 8; r++, o += step) {
                    if (in && r0 + r < rows) *reinterpret_cast<uint16_t *>(o) = (uint16_t)v[r];
                    if (both && r0 + r < rows) *reinterpret_cast<uint16_t *>(o + 2) = (uint16_t)(v[r] >> 16);
                }
            } else {
#pragma unroll
                for (int r = 0; r < 8; r++, o += step)
                    if (in && r0 + r < rows) *reinterpret_cast<uint32_t *>(o) = v[r];
            }
        }
        __syncwarp();
    }
}

// count<TN>() of a tile's features, from c_first on, of the 32 tokens of lane quarter q.
template <int TN, int SPLIT, int PAIR>
__device__ __forceinline__ void finish_tiles(const CUtensorMap &map_out, const Params &P, const Sums &S, int c_first, int q, int lane, uint32_t &gave_up)
{
    constexpr int COUNT = count<TN>(), PIECES = COUNT / 16, BUF = buffers<TN>();
    uint32_t it = 0;
    for (int tile = S.first; tile < P.tiles; tile += S.step, it++) {
        const int t0 = (tile % P.tiles_t * PAIR + S.t_rank) * TM, n0 = tile / P.tiles_t * TN;
        const uint32_t buf = it % BUF;
        uint32_t d[PIECES][16];
        mbar_wait_or_flag(S.acc_full + 8 * buf, (it / BUF) & 1, S.lost_at, gave_up);
        tc_fence_after();
        const bool any = t0 + 32 * q < P.B && c_first < TN;                // (the same for the warp's lanes)
        if (any) {
#pragma unroll
            for (int j = 0; j < PIECES; j++) tmem_start16(S.tmem + buf * TN + 16 * j, d[j]);
#pragma unroll
            for (int j = 0; j < PIECES; j++) tmem_wait16(d[j]);
        }
        // everything read: the buffer is the MMA warp's again
        tc_fence_before();
        __syncwarp();
        if (lane == 0 && !gave_up) {
            if (PAIR == 2) arrive_in_cluster(S.acc_empty + 8 * buf);
            else mbar_arrive(S.acc_empty + 8 * buf);
        }
        if (!any) continue;
        if constexpr (SPLIT > 1) {
            // the tile's sums over this CTA's columns: [128][TN] FP32 where the stages were (the last MMAs, which this warp has seen
            // end, were the last to read those); 16-byte pieces of a row exchanged so that the lanes of a quarter warp write different banks
            const int row = 32 * q + lane;
            if (t0 + row < P.B) {
#pragma unroll
                for (int j = 0; j < COUNT / 4; j++) {
                    const int piece = (c_first / 4 + j) ^ (lane & 7);
                    *reinterpret_cast<uint4 *>(S.sm + (row * TN + 4 * piece) * 4) = make_uint4(d[j / 4][j % 4 * 4], d[j / 4][j % 4 * 4 + 1], d[j / 4][j % 4 * 4 + 2], d[j / 4][j % 4 * 4 + 3]);
                }
            }
        } else {
            // through the warp's staging rows, 128 bytes (64 or 32 features) at a time, swizzled as the store's map says.  (In rows of 32 bytes the
            // copies out took 2.4 us for a tile of 256 features; 16384 x 512 at 2048 tokens 24 us instead of 15.)
            const int row = t0 + 32 * q, col = n0 + c_first;
            if (P.out_dtype == VPTQ_DTYPE_FP32) {
#pragma unroll
                for (int j = 0; j < PIECES; j += 2)
                    store_piece<true>(map_out, P, S, lane, row, col + 16 * j, [&](int c) {
                        const uint32_t *v = d[j + c / 4] + c % 4 * 4;
                        return make_uint4(v[0], v[1], v[2], v[3]);
                    });
            } else {
#pragma unroll
                for (int j = 0; j < PIECES; j += 4)
                    store_piece<false>(map_out, P, S, lane, row, col + 16 * j, [&](int c) {
                        uint32_t h[4];
#pragma unroll
                        for (int i = 0; i < 4; i++) h[i] = pair16(__uint_as_float(d[j + c / 2][c % 2 * 8 + 2 * i]), __uint_as_float(d[j + c / 2][c % 2 * 8 + 2 * i + 1]), P.out_dtype);
                        return make_uint4(h[0], h[1], h[2], h[3]);
                    });
            }
            // a lane that gave up went on without handing anything on; the warp's sums are no good whichever lane it was
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

// FEW: fewer than 128 tokens (whose part of a stage is not known here)
template <int TN, int SPLIT, int PAIR, bool FEW>
__global__ void __launch_bounds__(THREADS, 1)
linear_fp4_tcgen05_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_xs,
                          const __grid_constant__ CUtensorMap map_ws, const __grid_constant__ CUtensorMap map_out, const __grid_constant__ Params P)
{
    constexpr int RT = row_tiles<TN>(), BUF = buffers<TN>();
    // of a stage: activations, weight, their scales
    const uint32_t W_AT = FEW ? P.x_bytes : TM * KB_BYTES, SB = W_AT + weight_bytes<TN, PAIR>(), ST = FEW ? P.stages : stages<TN, PAIR>(TM * KB_BYTES), XS_AT = W_AT + TN / PAIR * KB_BYTES, WS_AT = XS_AT + SCALES;
    extern __shared__ __align__(1024) uint8_t sm[];
    __shared__ uint32_t tmem_slot, lost;                  // lost: a wait of this CTA gave up (of a pair: of either)
    const uint32_t base = smem_addr(sm), staging0 = base + ST * SB, bars = staging0 + FIXED_BYTES - BARRIERS;
    auto bar_full = [&](int s) { return bars + 8u * s; };
    auto bar_empty = [&](int s) { return bars + 8u * (MAX_STAGES + s); };
    auto bar_acc_full = [&](int b) { return bars + 8u * (2 * MAX_STAGES + b); };
    auto bar_acc_empty = [&](int b) { return bars + 8u * (2 * MAX_STAGES + 2 + b); };
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        lost = 0;
        for (uint32_t s = 0; s < ST; s++) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 1); }
        for (int b = 0; b < BUF; b++) { mbar_init(bar_acc_full(b), 1); mbar_init(bar_acc_empty(b), PAIR * ACC_WARPS); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc_all<PAIR>(smem_addr(&tmem_slot));
    if (warp == 0 && elect_one()) {
        prefetch_map(&map_w);
        prefetch_map(&map_x);
        if (PAIR == 2) { prefetch_map(&map_ws); prefetch_map(&map_xs); }
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
            uint32_t s = 0, round = 0;
            const uint32_t full0 = PAIR > 1 ? address_in(bar_full(0), 0) : bar_full(0);
            const int n_part = t_rank * (TN / PAIR);
            // the weight's part of a stage, and what the stage waits for; then the tokens'.  (One lane calls them.)
            auto scale_bytes = [&](int kb) { return (uint32_t)(min(CHUNKS, P.col_tiles - kb * CHUNKS) * FP4_TILE_BYTES); };
            auto load_weight = [&](uint32_t s, int kb, int n0) {
                const uint32_t at = base + s * SB, full = full0 + 8 * s;
                const int w_tile = n0 / FP4_TILE_ROWS * P.col_tiles + kb * CHUNKS;
                if constexpr (PAIR == 2) {
                    if (t_rank == 0) mbar_expect_tx(bar_full(s), PAIR * SB);
#pragma unroll
                    for (int r = 0; r < RT; r++) tma_load<PAIR>(at + WS_AT + r * SCALES, &map_ws, 0, w_tile + r * P.col_tiles, full);
                } else {
                    // scales as linear copies, of the tiles that there are: two maps fewer for the host to make (0.5 us of a call)
                    const uint32_t bytes = scale_bytes(kb), tiles = min(RT, P.row_tiles - n0 / FP4_TILE_ROWS);
                    mbar_expect_tx(full, W_AT + TN * KB_BYTES + (1 + tiles) * bytes);
#pragma unroll
                    for (int r = 0; r < RT; r++)
                        if (r < (int)tiles) bulk_load(at + WS_AT + r * SCALES, P.w_scale + (long long)(w_tile + r * P.col_tiles) * FP4_TILE_BYTES, bytes, full);
                }
                tma_load<PAIR>(at + W_AT, &map_w, kb * KB_BYTES, n0 + n_part, full);
            };
            auto load_tokens = [&](uint32_t s, int kb, int t0) {
                const uint32_t at = base + s * SB, full = full0 + 8 * s;
                const int x_tile = t0 / FP4_TILE_ROWS * P.col_tiles + kb * CHUNKS;
                if constexpr (PAIR == 2) tma_load<PAIR>(at + XS_AT, &map_xs, 0, x_tile, full);
                else bulk_load(at + XS_AT, P.x_scale + (long long)x_tile * FP4_TILE_BYTES, scale_bytes(kb), full);
                tma_load<PAIR>(at, &map_x, kb * KB_BYTES, t0, full);
            };
            // Behind the kernel that quantizes the tokens the weight need not wait for it.
            int begun = P.weight_early ? min((int)ST, kb1 - kb0) : 0;
            if (first >= P.tiles) begun = 0;
            for (int i = 0; i < begun; i++) {
                if (elect_one()) load_weight((uint32_t)i, kb0 + i, first / P.tiles_t * TN);
                __syncwarp();
            }
            pdl_wait();                                                        // (weight and activations may be the preceding kernel's)
            for (int tile = first; tile < P.tiles; tile += step) {
                const int t0 = (tile % P.tiles_t * PAIR + t_rank) * TM, n0 = tile / P.tiles_t * TN;
                for (int kb = kb0; kb < kb1; kb++, begun--) {
                    mbar_wait_or_flag(bar_empty(s), (round & 1) ^ 1u, lost_at, gave_up);
                    if (elect_one() && !gave_up) {
                        if (begun <= 0) load_weight(s, kb, n0);
                        load_tokens(s, kb, t0);
                    }
                    __syncwarp();
                    if (++s == ST) { s = 0; round++; }
                }
            }
        } else if (warp == 1) {
            // ---- scales to TMEM, then MMAs: e2m1 x e2m1 -> FP32, both K-major; of a pair, rank 0's over the memory of both ----
            constexpr uint32_t IDESC = (1u << 7) | (1u << 10) | ((uint32_t)(TN >> 3) << 17) | (1u << 23) | ((uint32_t)(PAIR * TM >> 4) << 24);
            const uint64_t a0 = make_smem_desc(base, 16, 1024, LAYOUT_SW128), b0 = make_smem_desc(base + W_AT, 16, 1024, LAYOUT_SW128);
            const uint64_t as0 = make_smem_desc(base + XS_AT, 16, 128, 0), bs0 = make_smem_desc(base + WS_AT, 16, 128, 0);
            uint32_t s = 0, round = 0, turn = 0, n = 0;
            pdl_wait();                                                        // (a wait's time does not begin before the preceding kernel has ended)
            for (int tile = first; tile < P.tiles && t_rank == 0; tile += step, n++) {
                const uint32_t buf = n % BUF, d = tmem + buf * TN;
                // where the tile's features begin in their first scale tile: four columns hold 128 rows, 32 in each
                const uint32_t inside = (uint32_t)(tile / P.tiles_t * TN) % FP4_TILE_ROWS / 32;
                mbar_wait_or_flag(bar_acc_empty(buf), ((n / BUF) & 1) ^ 1u, lost_at, gave_up);
                for (int kb = kb0; kb < kb1; kb++, turn ^= 1) {
                    mbar_wait_flagged(bar_full(s), round & 1, P.wait_limit, lost_at, gave_up);
                    tc_fence_after();
                    if (elect_one() && !gave_up) {
                        const uint64_t at = (uint64_t)((s * SB) >> 4);
                        const uint32_t xs = tmem + BUF * TN + turn * SCALE_COLS, ws = xs + 4 * CHUNKS;
                        const int steps = kb == P.kbs - 1 ? P.last_steps : STEPS;
                        // (with the next block's scales copied before these MMAs, a stage was held for one block longer: 8192 x 28672 at 2048 tokens 176 us, not 162)
#pragma unroll
                        for (int c = 0; c < CHUNKS; c++) {
                            if (2 * c >= steps) break;                         // (what lies behind the last columns is another row's)
                            copy_scales<PAIR>(xs + 4 * c, as0 + at + c * (FP4_TILE_BYTES >> 4));
#pragma unroll
                            for (int r = 0; r < RT; r++) copy_scales<PAIR>(ws + 4 * (c * RT + r), bs0 + at + (r * SCALES + c * FP4_TILE_BYTES >> 4));
                        }
#pragma unroll
                        for (int k = 0; k < STEPS; k++) {
                            if (k >= steps) break;
                            // (bytes 0 and 1, or 2 and 3, of a scale tile's words)
                            const uint32_t id = IDESC | (uint32_t)(k & 1) << 30 | (uint32_t)(k & 1) << 5;
                            mma_fp4<PAIR>(d, a0 + at + 2 * k, b0 + at + 2 * k, id, xs + 4 * (k / 2), ws + 4 * RT * (k / 2) + inside, kb > kb0 || k > 0);
                        }
                        commit<PAIR>(bar_empty(s));
                        if (kb == kb1 - 1) commit<PAIR>(bar_acc_full(buf));
                    }
                    __syncwarp();
                    if (++s == ST) { s = 0; round++; }
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
        const Sums S = {tmem + ((uint32_t)(32 * q) << 16) + share * count<TN>(), staging0 + w * STAGING, sm + ST * SB + w * STAGING, sm, lost_at,
                        bar_acc_full(0), PAIR > 1 ? address_in(bar_acc_empty(0), 0) : bar_acc_empty(0), first, step, t_rank};
        finish_tiles<TN, SPLIT, PAIR>(map_out, P, S, share * count<TN>(), q, lane, gave_up);
        report();
        if constexpr (SPLIT > 1) {
            cluster_sync();
            const uint32_t peer_lost = lane < SPLIT ? load_peer_word(lost_at, (uint32_t)lane) : 0u;       // (looked at below: no wait for it here)
            // rows of the tile that are tokens, dealt out over the ranks; four features a thread, the ranks' sums added in order
            const int t0 = first % P.tiles_t * TM, n0 = first / P.tiles_t * TN;
            constexpr int PIECES = TN / 4;
            const int all = min(TM, P.B - t0) * PIECES, i0 = (int)((long long)all * rank / SPLIT), i1 = (int)((long long)all * (rank + 1) / SPLIT);
            // (two ranks: several pieces' reads under way at a time, 2048 x 8192 at 300 tokens 10.0 -> 9.8 us; four ranks, whose shares are smaller: 6.9 -> 7.3, not taken)
            constexpr int TOGETHER = SPLIT == 2 ? 4 : 1, TAKERS = 32 * ACC_WARPS;
#pragma unroll 1
            for (int i = i0 + threadIdx.x - 32 * ACC_WARP0; i < i1; i += TAKERS * TOGETHER) {
                float4 v[TOGETHER][SPLIT];
#pragma unroll
                for (int u = 0; u < TOGETHER; u++) {
                    const int k = min(i + u * TAKERS, i1 - 1), row = k / PIECES, p = k % PIECES;
                    const uint32_t at = base + (uint32_t)(row * TN + 4 * (p ^ (row & 7))) * 4u;
#pragma unroll
                    for (int r = 0; r < SPLIT; r++) v[u][r] = load_peer(at, (uint32_t)r);
                }
#pragma unroll
                for (int u = 0; u < TOGETHER; u++) {
                    const int k = i + u * TAKERS, row = k / PIECES, col = n0 + 4 * (k % PIECES);
                    if (k >= i1) break;
                    float4 &t = v[u][0];
#pragma unroll
                    for (int r = 1; r < SPLIT; r++) { t.x += v[u][r].x; t.y += v[u][r].y; t.z += v[u][r].z; t.w += v[u][r].w; }
                    const long long o = (long long)(t0 + row) * P.M + col;
                    if (P.tma_out && col + 4 <= P.M) {                             // rows of 16-byte multiples: a thread's four values are aligned
                        if (P.out_dtype == VPTQ_DTYPE_FP32) *reinterpret_cast<float4 *>(reinterpret_cast<float *>(P.out) + o) = t;
                        else *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(P.out) + o) = make_uint2(pair16(t.x, t.y, P.out_dtype), pair16(t.z, t.w, P.out_dtype));
                    } else {
                        const float e[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
                        for (int c = 0; c < 4; c++)
                            if (col + c < P.M) store_out(P.out, o + c, e[c], P.out_dtype);
                    }
                }
            }
            __syncwarp();
            if (__any_sync(0xffffffffu, peer_lost != 0)) {                     // (the same for every warp, and for every rank: all of the tile)
                asm volatile("bar.sync 1, %0;" ::"n"(32 * ACC_WARPS) : "memory");
                for (int i = i0 + threadIdx.x - 32 * ACC_WARP0; i < i1; i += 32 * ACC_WARPS)
                    for (int k = 0; k < 4; k++) {
                        const int col = n0 + 4 * (i % PIECES) + k;
                        if (col < P.M) store_out(P.out, (long long)(t0 + i / PIECES) * P.M + col, __int_as_float(0x7FFFFFFF), P.out_dtype);
                    }
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

// scale tiles: rows of 512 bytes
bool map_scales(CUtensorMap *map, const uint8_t *p, int rows, int cols)
{
    const uint64_t tiles = (uint64_t)(fp4_scale_bytes(rows, cols) / FP4_TILE_BYTES);
    return encode_tensor_map(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, p, FP4_TILE_BYTES / 4, tiles, FP4_TILE_BYTES, 0, 0, FP4_TILE_BYTES / 4, CHUNKS, 1, CU_TENSOR_MAP_SWIZZLE_NONE);
}

template <int TN, int SPLIT, int PAIR, bool FEW>
cudaError_t run_as(const Fp4Linear &L, const Params &P0, cudaStream_t st)
{
    Params P = P0;
    const long long pitch = fp4_row_bytes(L.N), out_bytes = L.out_dtype == VPTQ_DTYPE_FP32 ? 4 : 2;
    CUtensorMap map_x, map_w, map_xs, map_ws, map_out;
    // (rows that are no tokens are not filled either: a fill with zeros takes as long as a load, and their sums are not read)
    const int x_rows = L.B < TM ? (L.B + 7) / 8 * 8 : TM;
    P.x_bytes = x_rows * KB_BYTES;
    P.stages = stages<TN, PAIR>(P.x_bytes);
    if (!encode_tensor_map(&map_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, L.x, pitch, L.B, pitch, 0, 0, KB_BYTES, x_rows, 1, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !encode_tensor_map(&map_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, L.w, pitch, L.M, pitch, 0, 0, KB_BYTES, TN / PAIR, 1, CU_TENSOR_MAP_SWIZZLE_128B) ||
        (PAIR == 2 && (!map_scales(&map_xs, L.x_scale, L.B, L.N) || !map_scales(&map_ws, L.w_scale, L.M, L.N))))
        return cudaErrorNotSupported;
    if (PAIR == 1) map_xs = map_ws = map_x;               // (not read)
    map_out = map_x;                                      // (not read unless tma_out)
    P.tma_out = L.M * out_bytes % 16 == 0 ? 1 : 0;
    if (P.tma_out &&
        !encode_tensor_map(&map_out, out_bytes == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, L.out, L.M, L.B, L.M * out_bytes, 0, 0, (uint32_t)(128 / out_bytes), 32, 1,
                           CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorNotSupported;
    P.tiles_t = ceil_div(L.B, PAIR * TM);
    P.tiles = P.tiles_t * ceil_div(L.M, TN);
    auto kern = linear_fp4_tcgen05_kernel<TN, SPLIT, PAIR, FEW>;
    constexpr int SMEM = SMEM_MAX, CLUSTER = SPLIT * PAIR;
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
    if (pdl_enabled("linear_fp4")) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        n++;
    }
    cfg.attrs = attr; cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kern, map_x, map_w, map_xs, map_ws, map_out, P);
}

template <int TN, int SPLIT, int PAIR>
cudaError_t run(const Fp4Linear &L, const Params &P, cudaStream_t st)
{
    if constexpr (PAIR == 1)
        if (L.B <= TM - 8) return run_as<TN, SPLIT, 1, true>(L, P, st);
    return run_as<TN, SPLIT, PAIR, false>(L, P, st);
}

template <int TN>
int resident_splits_of(int split)
{
    const void *kern = split == 2 ? (const void *)linear_fp4_tcgen05_kernel<TN, 2, 1, false> : split == 4 ? (const void *)linear_fp4_tcgen05_kernel<TN, 4, 1, false>
                                                                                                   : (const void *)linear_fp4_tcgen05_kernel<TN, 8, 1, false>;
    return max_resident_clusters(kern, split, THREADS, SMEM_MAX);
}
// split tiles that work at a time
int resident_splits(int tn, int split) { return tn == 64 ? resident_splits_of<64>(split) : resident_splits_of<128>(split); }

struct Choice { int tn, split, pair; };

// Tile width, split and pairs by estimated time.  A stage takes as long as its bytes take into shared memory, 113 to a nanosecond and SM (256 x 256 of a
// pair: 350 ns, 128 x 128: 300), or its MMAs, 280 ns for 256 features, and 250 at least; all of the weight takes as long as HBM needs for it.
// A tile ends with 0.5 us of 64 features, 0.7 of 128, 1.1 of 256 for its results (300 x 600 at 100 tokens: 3.8, 4.2, 6.6), a split one with 0.5 and
// 0.08 ns a sum more for the meeting (128 x 128 sums 1.8 us, 16 x 128 0.7).  Clusters of 8 CTAs: of those that the occupancy query promises half came at
// once (1024 x 8192 at 16 tokens: 16 clusters 8.4 us, 8 of tiles twice as wide 4.6).
// Pairs do not split: clusters of two or four pairs came to 16.9 us instead of 17.8 for 4096 x 14336 at 300 tokens, and nowhere else to less.
Choice choose(int M, int N, int B, int kbs)
{
    constexpr int WIDTHS = 3;
    const int widths[WIDTHS] = {256, 128, 64}, splits[4] = {1, 2, 4, 8};
    const int sms = device_sm_count();
    Choice best = {256, 1, 1};
    double best_time = 1e300;
    for (int pair = 1; pair <= 2; pair++)
        for (int i = 0; i < WIDTHS; i++)
            for (int j = 0; j < 4; j++) {
                const int tn = widths[i], split = splits[j];
                if (pair > 1 && (B <= TM || tn < 128)) continue;
                if (split > 1 && (tn > 128 || kbs < 2 * split || pair > 1)) continue;
                const long long tiles = (long long)ceil_div(B, pair * TM) * ceil_div(M, tn);
                if (split > 1 && tiles > resident_splits(tn, split) / (split == 8 ? 2 : 1)) continue;
                const long long waves = split > 1 ? 1 : (tiles + sms / pair - 1) / (sms / pair);
                const int bytes = (B < TM ? B : TM) * KB_BYTES + tn / pair * KB_BYTES + (tn > 128 ? 3 : 2) * SCALES;
                const double block = fmax(bytes / 113.0, fmax(280.0 / 256 * tn, 250));
                const double time = waves * (ceil_div(kbs, split) * block + 300 + 3 * tn + (split > 1 ? 500 + 0.08 * (B < TM ? B : TM) * tn : 0)), hbm = M * (N * (17.0 / 32)) / 6000;
                const double longer = fmax(time, hbm) + 0.01 * time;
                if (longer < best_time) { best_time = longer; best = {tn, split, pair}; }
            }
    return best;
}

}  // namespace

cudaError_t launch_linear_fp4_tcgen05(const Fp4Linear &L, int *status, bool early, cudaStream_t st)
{
    Params P;
    P.M = L.M; P.B = L.B; P.kbs = ceil_div(L.N, KB);
    P.last_steps = ceil_div(L.N - (P.kbs - 1) * KB, 64);
    P.col_tiles = ceil_div(L.N, FP4_TILE_COLS); P.row_tiles = ceil_div(L.M, FP4_TILE_ROWS);
    P.x_scale = L.x_scale; P.w_scale = L.w_scale;
    P.out = L.out; P.out_dtype = L.out_dtype; P.status = status;
    P.wait_limit = wait_limit();
    P.weight_early = early ? 1 : 0;
    P.tiles_t = P.tiles = P.tma_out = P.x_bytes = P.stages = 0;
    const Choice c = choose(L.M, L.N, L.B, P.kbs);
    if (c.pair == 2) switch (c.tn) {
        case 256: return run<256, 1, 2>(L, P, st);
        default: return run<128, 1, 2>(L, P, st);
        }
    switch (c.tn * 10 + c.split) {
    case 2561: return run<256, 1, 1>(L, P, st);
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
