// out = x W^T for a few tokens over an e2m1 weight, in one kernel: the activations are quantized by the CTAs that multiply by them.
//
// What counts is the weight's way from HBM; the products are the tensor cores' (tcgen05.mma, kind::mxf4, as in linear_fp4_tcgen05.cu), so that no
// code of the weight passes through a register.  The tokens are rows of the MMA's first operand, of whose 128 rows only those that are tokens lie in
// shared memory: the others are whatever follows there, and sums of lanes that nobody reads.
// A CTA takes some groups of 32 features (a scale tile's columns of TMEM hold 32 rows each), at most seven at a time, dealt out evenly so that all
// SMs load; a layer of fewer groups than SMs has its columns split over the CTAs of a cluster, which send each other their sums: every CTA adds
// up its share of the results, in rank order.
// Warps by role: 0 loads the weight and its scales (TMA) through a ring of stages of 256 columns, 1 copies scales to TMEM and issues the
// MMAs, the others quantize the activations (the rule of fp4_quantize.cu; e2m1 activations: copy them) block by block into the layout of the operand,
// where they stay; two of them read the sums in the end.
// Every wait is bounded; sums of a CTA in which one gave up are NaN, and the workspace's status word is set.
#include "fp4.cuh"
#include "fp4_tcgen05.cuh"
#include "tcgen05_pair.cuh"

namespace vptq {

namespace {

using namespace tc;

constexpr int KB = 256, KB_BYTES = KB / 2;                // columns of a block: a swizzled row of 128 bytes
constexpr int STEPS = KB / 64, CHUNKS = KB / FP4_TILE_COLS;            // MMAs, and scale tiles of 128 rows, along a block
// Features of a group, groups of a pass at most.  An MMA's features begin at a multiple of 64: scale addresses in TMEM are even columns.  A pass that
// begins at an odd group leaves the place of the group before it unused, in shared memory and among the sums.
constexpr int GROUP = 32, GROUPS = 7;
constexpr int GROUP_BYTES = GROUP * KB_BYTES, SCALES = CHUNKS * FP4_TILE_BYTES;
constexpr int WARPS = 12, THREADS = 32 * WARPS, X_WARP0 = 2, SUM_WARP0 = 4, SUM_WARP1 = 8;      // (the warps that may read lanes 0..31 of TMEM)
constexpr int X_HALVES = 2 * (WARPS - X_WARP0);
constexpr int MAX_STAGES = 16;
constexpr int MIN_RING = 16 * 1024;                       // an MMA reads 128 rows from its block of activations on
constexpr int SMEM_MAX = 232448 - 1024;                  // (the static part takes a multiple of the dynamic part's alignment)
// Two CTAs fit on an SM where their shared memory does: the next launch's are made ready beside these.  Together they never ask for more TMEM than
// there is: one that wants more than half of its 512 columns has an SM to itself (CTAs of two clusters could wait for each other's).
constexpr int HALF_SMEM = 113 * 1024, WHOLE_SMEM = 116 * 1024;

struct Params {
    int M, N, B, kbs, last_steps, col_tiles;
    int groups, split;                                    // of the layer; CTAs of a cluster
    int pass_groups, row_tiles;                           // groups and scale tiles that a stage has room for
    int stages, x_rows;                                   // x_rows: tokens, rounded up to 8
    int tmem_cols;
    const void *x;
    const uint8_t *x_scale;
    void *out;
    int out_dtype, wide_out;                              // wide_out: rows of `out` are 16-byte aligned
    int *status;
    unsigned long long wait_limit;
};

__device__ __forceinline__ void mma(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t a_scale, uint32_t b_scale, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(a_scale), "r"(b_scale), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc)
{
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void store_peer4(uint32_t addr, uint32_t rank, float4 v)
{
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(address_in(addr, rank)), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

// sixteen columns of a token: values that are to be quantized, or codes and their scale byte
template <int DT, bool VEC> struct Item { Sixteen<DT, VEC> v; };
template <> struct Item<VPTQ_DTYPE_E2M1, true> { uint2 q; uint32_t b; };

template <int DT, bool VEC>
__device__ __forceinline__ void load_item(const Params &P, int row, int c, Item<DT, VEC> &e)
{
    if constexpr (DT == VPTQ_DTYPE_E2M1) {
        const long long pitch = (long long)((P.N + FP4_BLOCK - 1) / FP4_BLOCK) * (FP4_BLOCK / 2);
        e.q = make_uint2(0, 0);
        e.b = 0;
        if (row < P.B && c / 2 < pitch) {
            e.q = __ldg(reinterpret_cast<const uint2 *>(reinterpret_cast<const uint8_t *>(P.x) + row * pitch + c / 2));
            e.b = __ldg(P.x_scale + (long long)(c / FP4_TILE_COLS) * FP4_TILE_BYTES + fp4_scale_at(row, c / FP4_BLOCK % 4));
        }
    } else {
        e.v = load_sixteen<DT, VEC>(reinterpret_cast<const uint8_t *>(P.x) + (long long)row * P.N * Act<DT>::BYTES, row < P.B ? c : P.N, P.N);
    }
}
// its codes and scale byte; for a whole warp
template <int DT, bool VEC>
__device__ __forceinline__ uint2 codes_of(const Item<DT, VEC> &e, int n, uint32_t &b)
{
    if constexpr (DT == VPTQ_DTYPE_E2M1) {
        b = e.b;
        return e.q;
    } else {
        b = fp4_pair_scale(magnitude(e.v));
        return fp4_codes16(e.v, b, n);
    }
}

template <int DT, bool VEC>
__global__ void __launch_bounds__(THREADS, 2)
linear_fp4_few_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_ws, const __grid_constant__ Params P)
{
    extern __shared__ __align__(1024) uint8_t sm[];
    __shared__ uint32_t tmem_slot, lost;                  // lost: a wait of this CTA gave up
    __shared__ __align__(8) uint64_t barriers[2 * MAX_STAGES + 2];
    // shared memory: activations by block, stages, the activations' scales by block, what the cluster's CTAs send, a barrier for every block
    const int rank = P.split > 1 ? (int)cluster_rank() : 0, cluster = (int)blockIdx.x / P.split, clusters = (int)gridDim.x / P.split;
    const int kb0 = (int)((long long)P.kbs * rank / P.split), kb1 = (int)((long long)P.kbs * (rank + 1) / P.split), blocks = kb1 - kb0;
    const int most_blocks = (P.kbs + P.split - 1) / P.split;
    const uint32_t x_block = (uint32_t)P.x_rows * KB_BYTES, xs_chunk = (uint32_t)P.x_rows * 16u;
    const uint32_t places = P.pass_groups + 1, stage_bytes = places * GROUP_BYTES + (uint32_t)P.row_tiles * SCALES;
    const uint32_t base = smem_addr(sm), ring = base + (most_blocks * x_block + 1023u & ~1023u), xs0 = ring + P.stages * stage_bytes;
    const uint32_t sums = xs0 + (most_blocks * CHUNKS * xs_chunk + FP4_TILE_BYTES + 15u & ~15u);
    const uint32_t x_bars = sums + (P.split > 1 ? (uint32_t)(P.x_rows * P.pass_groups * GROUP * 4 + 16 * P.split) : 0u);
    const uint32_t bars = smem_addr(barriers);
    auto bar_full = [&](int s) { return bars + 8u * s; };
    auto bar_empty = [&](int s) { return bars + 8u * (MAX_STAGES + s); };
    const uint32_t bar_acc_full = bars + 8u * 2 * MAX_STAGES, bar_acc_empty = bar_acc_full + 8;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        lost = 0;
        for (int s = 0; s < P.stages; s++) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 1); }
        mbar_init(bar_acc_full, 1);
        mbar_init(bar_acc_empty, 2);
    }
    for (int i = threadIdx.x; i < blocks; i += THREADS) mbar_init(x_bars + 8 * i, P.x_rows);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_slot)), "r"(P.tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    if (P.split > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");       // (waited for before anything is sent)
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    pdl_launch_dependents();

    // this cluster's groups, in passes of nearly the same number
    const int g_first = (int)((long long)P.groups * cluster / clusters), g_end = (int)((long long)P.groups * (cluster + 1) / clusters);
    const int passes = (g_end - g_first + P.pass_groups - 1) / P.pass_groups;
    auto pass_begin = [&](int p) { return g_first + (int)((long long)(g_end - g_first) * p / passes); };
    const uint32_t lost_at = smem_addr(&lost);
    uint32_t gave_up = 0;
    pdl_wait();                                                                // (weight and activations may be the preceding kernel's, and it may read the result's memory)

    if (warp == 0) {
        // ---- loads ----
        uint32_t s = 0, round = 0;
        for (int p = 0; p < passes; p++) {
            const int g0 = pass_begin(p), n = pass_begin(p + 1) - g0, tiles = (g0 % 4 + n + 3) / 4;
            for (int kb = kb0; kb < kb1; kb++) {
                mbar_wait_or_flag(bar_empty(s), (round & 1) ^ 1u, lost_at, gave_up);
                if (elect_one() && !gave_up) {
                    const uint32_t at = ring + s * stage_bytes, full = bar_full(s);
                    mbar_expect_tx(full, (uint32_t)(n * GROUP_BYTES + tiles * SCALES));
                    for (int i = 0; i < n; i++) tma_load_2d(at + (g0 % 2 + i) * GROUP_BYTES, &map_w, kb * KB_BYTES, (g0 + i) * GROUP, full);
                    for (int i = 0; i < tiles; i++)
                        tma_load_2d(at + places * GROUP_BYTES + i * SCALES, &map_ws, 0, (g0 / 4 + i) * P.col_tiles + kb * CHUNKS, full);
                }
                __syncwarp();
                if (++s == (uint32_t)P.stages) { s = 0; round++; }
            }
        }
    } else if (warp == 1) {
        // ---- scales to TMEM, then MMAs ----
        const uint64_t a0 = make_smem_desc(base, 16, 1024, LAYOUT_SW128), b0 = make_smem_desc(ring, 16, 1024, LAYOUT_SW128);
        const uint64_t as0 = make_smem_desc(xs0, 16, 128, 0), bs0 = make_smem_desc(ring + places * GROUP_BYTES, 16, 128, 0);
        uint32_t s = 0, round = 0, turn = 0;
        for (int p = 0; p < passes; p++) {
            const int g0 = pass_begin(p), n = pass_begin(p + 1) - g0;
            const uint32_t tiles = (uint32_t)(g0 % 4 + n + 3) / 4, inside = g0 % 4 / 2 * 2;
            const uint32_t idesc = (1u << 7) | (1u << 10) | ((uint32_t)((g0 % 2 + n) * GROUP >> 3) << 17) | (1u << 23) | ((128u >> 4) << 24);
            mbar_wait_or_flag(bar_acc_empty, (p & 1) ^ 1u, lost_at, gave_up);
            for (int kb = kb0; kb < kb1; kb++, turn ^= 1) {
                if (p == 0) mbar_wait_flagged(x_bars + 8 * (kb - kb0), 0, P.wait_limit, lost_at, gave_up);
                mbar_wait_flagged(bar_full(s), round & 1, P.wait_limit, lost_at, gave_up);
                tc_fence_after();
                if (elect_one() && !gave_up) {
                    const uint64_t at = (uint64_t)(s * stage_bytes >> 4), xa = (uint64_t)((kb - kb0) * x_block >> 4), xsa = (uint64_t)((kb - kb0) * CHUNKS * xs_chunk >> 4);
                    const uint32_t xs = tmem + places * GROUP + turn * 32, ws = xs + 4 * CHUNKS;
                    const int steps = kb == P.kbs - 1 ? P.last_steps : STEPS;
#pragma unroll
                    for (int c = 0; c < CHUNKS; c++) {
                        if (2 * c >= steps) break;                             // (what lies behind the last columns is another row's)
                        copy_scales(xs + 4 * c, as0 + xsa + c * (xs_chunk >> 4));
                        for (uint32_t r = 0; r < tiles; r++) copy_scales(ws + 4 * (c * tiles + r), bs0 + at + (r * SCALES + c * FP4_TILE_BYTES >> 4));
                    }
#pragma unroll
                    for (int k = 0; k < STEPS; k++) {
                        if (k >= steps) break;
                        const uint32_t id = idesc | (uint32_t)(k & 1) << 30 | (uint32_t)(k & 1) << 5;
                        mma(tmem, a0 + xa + 2 * k, b0 + at + 2 * k, id, xs + 4 * (k / 2), ws + 4 * tiles * (k / 2) + inside, kb > kb0 || k > 0);
                    }
                    umma_commit(bar_empty(s));
                    if (kb == kb1 - 1) umma_commit(bar_acc_full);
                }
                __syncwarp();
                if (++s == (uint32_t)P.stages) { s = 0; round++; }
            }
        }
    } else {
        // ---- activations: half a warp takes a token's 256 columns ----
        if (blockIdx.x == 0 && threadIdx.x == 32 * X_WARP0) *P.status = 0;
        const int l = lane & 15, half = 2 * (warp - X_WARP0) + (lane >> 4), items = blocks * P.x_rows;
        int kb = half / P.x_rows, row = half - kb * P.x_rows;
        auto next = [&](int &kb, int &row) {
            row += X_HALVES;
            while (row >= P.x_rows) { row -= P.x_rows; kb++; }
        };
        Item<DT, VEC> e;
        load_item<DT, VEC>(P, row, kb < blocks ? (kb0 + kb) * KB + 16 * l : KB * P.kbs, e);
        for (int i = half - (lane >> 4); i < items; i += X_HALVES) {          // (a warp's halves run the same number of rounds: shuffles)
            Item<DT, VEC> e2;
            int kb2 = kb, row2 = row;
            next(kb2, row2);
            load_item<DT, VEC>(P, row2, kb2 < blocks ? (kb0 + kb2) * KB + 16 * l : KB * P.kbs, e2);
            uint32_t b;
            const uint2 q = codes_of<DT, VEC>(e, P.N - ((kb0 + kb) * KB + 16 * l), b);
            if (kb < blocks) {
                // 128-byte swizzle: the 16-byte pieces of a row are exchanged by the row's place among eight
                const uint32_t at = base + kb * x_block + row * KB_BYTES + ((l / 2 ^ row & 7) << 4) + (l & 1) * 8;
                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(q.x), "r"(q.y) : "memory");
                if ((l & 1) == 0) asm volatile("st.shared.u8 [%0], %1;" ::"r"(xs0 + (kb * CHUNKS + l / 8) * xs_chunk + row * 16 + l / 2 % 4), "r"(b) : "memory");
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            __syncwarp();
            if (l == 0 && kb < blocks) mbar_arrive(x_bars + 8 * kb);
            e = e2; kb = kb2; row = row2;
        }
        __syncwarp();
    }
    __syncwarp();
    if (P.split > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");          // the cluster's CTAs have begun
    const bool sums_up = warp == SUM_WARP0 || warp == SUM_WARP1;
    for (int p = 0; p < passes; p++) {
        const int g0 = pass_begin(p), n = pass_begin(p + 1) - g0, m0 = g0 * GROUP, cols = n * GROUP;
        if (sums_up) {
            mbar_wait_or_flag(bar_acc_full, p & 1, lost_at, gave_up);
            tc_fence_after();
            // (a lane that gave up, here or in another warp before this one was woken, leaves NaN)
            const bool bad = __any_sync(0xffffffffu, gave_up != 0 || load_word(lost_at) != 0);
            for (int c = warp == SUM_WARP0 ? 0 : 16; c < cols; c += 32) {
                uint32_t d[16];
                __syncwarp();
                tmem_start16(tmem + g0 % 2 * GROUP + c, d);
                tmem_wait16(d);
                if (bad)
#pragma unroll
                    for (int i = 0; i < 16; i++) d[i] = 0x7FFFFFFFu;
                if (lane >= P.B) continue;
                if (P.split > 1) {
                    // pieces of four results, token by token, are dealt out over the ranks; a rank's are side by side for every sender
                    const int all = P.B * (cols / 4);
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const int piece = lane * (cols / 4) + c / 4 + i, owner = (int)((long long)(piece + 1) * P.split - 1) / all;
                        const int first = (int)((long long)all * owner / P.split), count = (int)((long long)all * (owner + 1) / P.split) - first;
                        store_peer4(sums + (uint32_t)(rank * count + piece - first) * 16u, (uint32_t)owner,
                                    make_float4(__uint_as_float(d[4 * i]), __uint_as_float(d[4 * i + 1]), __uint_as_float(d[4 * i + 2]), __uint_as_float(d[4 * i + 3])));
                    }
                } else if (P.wide_out && m0 + c + 16 <= P.M) {
                    const long long o = (long long)lane * P.M + m0 + c;
                    if (P.out_dtype == VPTQ_DTYPE_FP32) {
#pragma unroll
                        for (int i = 0; i < 4; i++) reinterpret_cast<uint4 *>(reinterpret_cast<float *>(P.out) + o)[i] = make_uint4(d[4 * i], d[4 * i + 1], d[4 * i + 2], d[4 * i + 3]);
                    } else {
                        uint32_t h[8];
#pragma unroll
                        for (int i = 0; i < 8; i++) h[i] = pair16(__uint_as_float(d[2 * i]), __uint_as_float(d[2 * i + 1]), P.out_dtype);
#pragma unroll
                        for (int i = 0; i < 2; i++) reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(P.out) + o)[i] = make_uint4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; i++)
                        if (m0 + c + i < P.M) store_out(P.out, (long long)lane * P.M + m0 + c + i, __uint_as_float(d[i]), P.out_dtype);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0 && !gave_up) mbar_arrive(bar_acc_empty);
        }
        if (P.split > 1) {                                                     // (one pass)
            __syncwarp();
            cluster_sync();
            const int all = P.B * (cols / 4), first = (int)((long long)all * rank / P.split), count = (int)((long long)all * (rank + 1) / P.split) - first;
            for (int i = threadIdx.x; i < count; i += THREADS) {
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int r = 0; r < P.split; r++) {
                    float4 a;
                    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(a.x), "=f"(a.y), "=f"(a.z), "=f"(a.w) : "r"(sums + (uint32_t)(r * count + i) * 16u) : "memory");
                    v.x += a.x; v.y += a.y; v.z += a.z; v.w += a.w;
                }
                const int token = (first + i) / (cols / 4), m = m0 + (first + i - token * (cols / 4)) * 4;
                const long long o = (long long)token * P.M + m;
                const float t[4] = {v.x, v.y, v.z, v.w};
                if (P.wide_out && m + 4 <= P.M) {
                    if (P.out_dtype == VPTQ_DTYPE_FP32) *reinterpret_cast<float4 *>(reinterpret_cast<float *>(P.out) + o) = v;
                    else *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(P.out) + o) = make_uint2(pair16(v.x, v.y, P.out_dtype), pair16(v.z, v.w, P.out_dtype));
                } else {
                    for (int k = 0; k < 4; k++)
                        if (m + k < P.M) store_out(P.out, o + k, t[k], P.out_dtype);
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (*reinterpret_cast<volatile uint32_t *>(&lost)) {
        let_copies_land();
        if (threadIdx.x == 0) atomicExch(P.status, VPTQ_E_TIMEOUT);            // (long after the word was cleared)
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(P.tmem_cols) : "memory");
    }
}

// ---- host side ----------------------------------------------------------------------------------------

struct Plan {
    int split, clusters, pass_groups, row_tiles, stages, tmem_cols;
    size_t smem;
};

// what a CTA needs beside its stages
size_t fixed_bytes(int B, int kbs, int split, int pass_groups)
{
    const int x_rows = (B + 7) / 8 * 8, blocks = ceil_div(kbs, split);
    size_t n = ((size_t)blocks * x_rows * KB_BYTES + 1023) / 1024 * 1024 + ((size_t)blocks * CHUNKS * x_rows * 16 + FP4_TILE_BYTES + 15) / 16 * 16;
    if (split > 1) n += (size_t)x_rows * pass_groups * GROUP * 4 + 16 * split;
    return n + 8 * (size_t)blocks;
}

// Split, passes and stages by estimated time.
bool make_plan(int M, int B, int kbs, Plan *best)
{
    const int groups = ceil_div(M, GROUP), sms = device_sm_count();
    double best_cost = 1e300;
    for (int split = 1; split <= 8; split *= 2) {
        if (split > 1 && kbs < 2 * split) continue;
        int room = sms / split;                                                // clusters that work at a time
        if (split > 1) {
            const int fit = max_resident_clusters(reinterpret_cast<const void *>(linear_fp4_few_kernel<VPTQ_DTYPE_FP16, true>), split, THREADS, SMEM_MAX);
            if (fit < 1) continue;
            if (fit < room) room = fit;
        }
        Plan p;
        p.split = split;
        p.clusters = groups < room ? groups : room;
        const int most = ceil_div(groups, p.clusters);
        if (split > 1 && most > GROUPS) continue;
        const int passes = ceil_div(most, GROUPS);
        p.pass_groups = ceil_div(most, passes);
        p.row_tiles = (p.pass_groups + 3 + 3) / 4;                             // (a pass begins anywhere in a scale tile)
        const size_t stage = (size_t)(p.pass_groups + 1) * GROUP_BYTES + (size_t)p.row_tiles * SCALES, fixed = fixed_bytes(B, kbs, split, p.pass_groups);
        const int blocks = ceil_div(kbs, split);
        // as many stages as there are blocks, within half of an SM's memory if that is 64 KB of them, else within all of it
        auto fit = [&](size_t limit) { return limit > fixed ? (int)((limit - fixed) / stage) : 0; };
        int stages = fit(HALF_SMEM);
        if (stages < passes * blocks && stages * stage < 64 * 1024) stages = fit(SMEM_MAX);
        if (stages > MAX_STAGES) stages = MAX_STAGES;
        if (stages > passes * blocks) stages = passes * blocks;
        while (stages * stage < (size_t)MIN_RING) stages++;                    // (never beyond MAX_STAGES: a stage has 9 KB at least)
        if (stages < 1 || fixed + stages * stage > (size_t)SMEM_MAX || (stages < 2 && passes * blocks > 1)) continue;
        p.stages = stages;
        p.smem = fixed + stages * stage;
        p.tmem_cols = 32;
        while (p.tmem_cols < (p.pass_groups + 1) * GROUP + 64) p.tmem_cols *= 2;
        if (p.tmem_cols > 256 && p.smem < (size_t)WHOLE_SMEM) p.smem = WHOLE_SMEM;
        const double cost = (double)most * blocks + (split > 1 ? 8 : 0);       // groups of features by blocks of columns, 0.1 us each; the meeting 0.8 us
        if (cost < best_cost) { best_cost = cost; *best = p; }
    }
    return best_cost < 1e300;
}

template <int DT, bool VEC>
cudaError_t run(const Fp4Linear &L, const Plan &p, const Params &P, cudaStream_t st)
{
    CUtensorMap map_w, map_ws;
    const long long pitch = fp4_row_bytes(L.N);
    const uint64_t tiles = (uint64_t)(fp4_scale_bytes(L.M, L.N) / FP4_TILE_BYTES);
    if (!encode_tensor_map(&map_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, L.w, pitch, L.M, pitch, 0, 0, KB_BYTES, GROUP, 1, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !encode_tensor_map(&map_ws, CU_TENSOR_MAP_DATA_TYPE_UINT32, L.w_scale, FP4_TILE_BYTES / 4, tiles, FP4_TILE_BYTES, 0, 0, FP4_TILE_BYTES / 4, CHUNKS, 1,
                           CU_TENSOR_MAP_SWIZZLE_NONE))
        return cudaErrorNotSupported;
    auto kern = linear_fp4_few_kernel<DT, VEC>;
    const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void *>(kern), SMEM_MAX);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.clusters * p.split));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = p.smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (p.split > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)p.split; attr[n].val.clusterDim.y = 1; attr[n].val.clusterDim.z = 1;
        n++;
    }
    if (pdl_enabled("linear_fp4")) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        n++;
    }
    cfg.attrs = attr; cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kern, map_w, map_ws, P);
}

}  // namespace

bool linear_fp4_few_takes(int M, int N, int B)
{
    Plan p;
    return B <= FP4_FEW_MAX_B && make_plan(M, B, ceil_div(N, KB), &p);
}

cudaError_t launch_linear_fp4_few(const Fp4Linear &L, int *status, cudaStream_t st)
{
    Plan p;
    const int kbs = ceil_div(L.N, KB);
    if (L.B > FP4_FEW_MAX_B || !make_plan(L.M, L.B, kbs, &p)) return cudaErrorNotSupported;
    Params P;
    P.M = L.M; P.N = L.N; P.B = L.B; P.kbs = kbs;
    P.last_steps = ceil_div(L.N - (kbs - 1) * KB, 64);
    P.col_tiles = ceil_div(L.N, FP4_TILE_COLS);
    P.groups = ceil_div(L.M, GROUP); P.split = p.split;
    P.pass_groups = p.pass_groups; P.row_tiles = p.row_tiles; P.stages = p.stages; P.x_rows = (L.B + 7) / 8 * 8; P.tmem_cols = p.tmem_cols;
    P.x = L.x; P.x_scale = L.x_scale; P.out = L.out; P.out_dtype = L.out_dtype;
    P.wide_out = (long long)L.M * (L.out_dtype == VPTQ_DTYPE_FP32 ? 4 : 2) % 16 == 0 ? 1 : 0;
    P.status = status; P.wait_limit = wait_limit();
    const bool vec = (reinterpret_cast<uintptr_t>(L.x) & 15u) == 0 && L.N % 8 == 0;
    switch (L.x_dtype) {
    case VPTQ_DTYPE_E2M1: return run<VPTQ_DTYPE_E2M1, true>(L, p, P, st);
    case VPTQ_DTYPE_FP16: return vec ? run<VPTQ_DTYPE_FP16, true>(L, p, P, st) : run<VPTQ_DTYPE_FP16, false>(L, p, P, st);
    default: return vec ? run<VPTQ_DTYPE_BF16, true>(L, p, P, st) : run<VPTQ_DTYPE_BF16, false>(L, p, P, st);
    }
}

}  // namespace vptq
