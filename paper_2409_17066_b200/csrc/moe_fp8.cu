// A mixture-of-experts layer for a few tokens over experts in e4m3 with 128 x 128 block scales, in two kernels:
//   logits = x Wr^T, p = softmax(logits), the k largest logits of a token (equal ones: the lowest expert) with weights p, or p divided
//   by the chosen ones' sum;  h = silu(x Wg^T) * (x Wu^T) per token and choice;  out = sum over the choices of weight * (h Wd^T).
//
// moe_gate_up_kernel: clusters of four CTAs quantize x and compute all logits, a quarter each, and every CTA makes the choices and the
// list of experts in use by itself: no wait for another cluster and no launch for the router.  Then 128 columns of h of an expert in
// use at a time are a cluster's, 32 gate and 32 up rows a CTA's: a warp takes every sixteenth 128-column block of them into a stage of
// its own (as in linear_fp8_decode.cu), multiplies it with up to 8 of the expert's tokens (fp8_mma.cuh), the warps' sums meet in shared
// memory, and the four CTAs exchange the largest magnitude of their 32 columns, so that h leaves as e4m3 with its scale.
// moe_down_kernel: a CTA owns 16 or 32 rows of the result; its warps share the blocks of all the experts in use; per expert a warp adds
// weight * sums to a slot of its own for each token, and the slots are added in warp order.  No atomics: a result does not depend on
// timing.
// Bound by HBM: the weights of the experts in use, each once (once for every 8 of its tokens; 2 of 8 experts of 4096 -> 14336 for 8 tokens:
// 224 to 253 us from one device to another, 5.7 and 5.4 TB/s in the two kernels); for one token of small experts (8 of 64 of 2048 -> 1024: 27 us) by the way through
// router, two launches and two reductions.  Quantizing x and h where they are multiplied cost 250 instructions a block,
// more than everything else in the loops together.
// Every wait is bounded; a CTA of the first kernel, or a warp of the second, whose wait gives up leaves NaN from there on.
#include "fp8_mma.cuh"
#include "moe_fp8.cuh"
#include "tcgen05_ptx.cuh"
#include "tma_2d.cuh"

namespace vptq {

namespace {

using namespace tc;

constexpr int GROUP = 16, GROUP_BYTES = GROUP * FP8_BLOCK;
constexpr int WARPS = 16, THREADS = 32 * WARPS;
constexpr int CLUSTER = 4;
constexpr int UNITS = 2;                                  // of a pass: 16 gate and 16 up rows each
constexpr int UP_GROUPS = 2 * UNITS;
constexpr int TOKENS = 8;                                 // of an expert at a time
constexpr int MAX_ENTRIES = MOE_MAX_TOKENS * MOE_MAX_TOP;
constexpr int DOWN_GROUPS = 2;                            // groups of a CTA's pass of the down kernel

// The experts in use, up to 8 of an expert's (token, choice) pairs to an entry; pair = token * top + choice.
struct Plan {
    int entries;
    int pad[3];
    float weight[MAX_ENTRIES];                            // of every pair
    int16_t expert[MAX_ENTRIES];
    int16_t count[MAX_ENTRIES];
    int16_t pair[MAX_ENTRIES][TOKENS];
};

struct Params {
    MoeFp8 L;
    Plan *plan;            // in the workspace, as are:
    uint8_t *hq;           // h: [T * top][hq_pitch] e4m3 and [T * top][ceil(inner / 128)] scales
    float *hs;
    uint8_t *xq;           // x, a copy for every cluster: [T][xq_pitch] e4m3 and [T][ceil(hidden / 128)] scales
    float *xs;
    int hq_pitch, xq_pitch;
    int down_groups;       // groups of a pass of the down kernel
    int down_passes, down_run_shift;
    unsigned long long wait_limit;
};

// a lane's share of one token's e4m3 values in one block, written by this kernel's cluster or by the kernel before; row: null for zeros
__device__ __forceinline__ TokenRaw<VPTQ_DTYPE_E4M3, true> load_e4m3(const uint8_t *row, int t, int kb, int pitch)
{
    TokenRaw<VPTQ_DTYPE_E4M3, true> r;
    const int c0 = kb * FP8_BLOCK + 16 * t;
#pragma unroll
    for (int c = 0; c < 2; c++) r.q[c] = row != nullptr && c0 + 64 * c < pitch ? __ldcg(reinterpret_cast<const uint4 *>(row + c0 + 64 * c)) : make_uint4(0, 0, 0, 0);
    return r;
}

__device__ __forceinline__ uint4 load_shared16(uint32_t a)
{
    uint4 q;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(a));
    return q;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void store_peer(float *at, uint32_t rank, float v)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(at)), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory");
}

// this cluster's copy of x in e4m3: a half warp a block, as in fp8_quantize.cu
template <int DT, bool VEC>
__device__ __forceinline__ void quantize_tokens(const MoeFp8 &L, uint8_t *xq, float *xs, int pitch, uint32_t rank)
{
    const int kbs = (L.hidden + FP8_BLOCK - 1) / FP8_BLOCK, lane = threadIdx.x & 15, half = (threadIdx.x >> 4) & 1;
    for (int b0 = ((int)rank * THREADS + (int)threadIdx.x >> 4) - half; b0 < L.T * kbs; b0 += CLUSTER * THREADS / 16) {      // (whole warps)
        const int block = b0 + half, token = block / kbs, kb = block % kbs, c = kb * FP8_BLOCK + lane * 8;
        const bool in = token < L.T;
        const Eight<DT, VEC> v = load_eight<DT, VEC>(reinterpret_cast<const uint8_t *>(L.x) + (long long)(in ? token : 0) * L.hidden * 2, in ? c : L.hidden, L.hidden);
        uint32_t m = magnitude(v);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        const Fp8Scale s = fp8_scale(__uint_as_float(m));
        if (in) {
            store_eight(xq + (long long)token * pitch, pitch, c, L.hidden, v, s.factor);
            if (lane == 0) xs[block] = s.scale;
        }
    }
}

// ... counted on a barrier of the same CTA when it has arrived
__device__ __forceinline__ void store_peer_async(float *at, uint32_t bar, uint32_t rank, float v)
{
    uint32_t a, b;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(at)), "r"(rank));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(b) : "r"(bar), "r"(rank));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(a), "r"(__float_as_uint(v)), "r"(b) : "memory");
}

// One warp: the products of an expert's router row with N tokens over columns [c0, c1); `ahead` loads of each row in flight.
template <int DT, bool VEC, int N>
__device__ __forceinline__ void router_products(const uint8_t *w, const uint8_t *x, long long row_bytes, int last_token, int c0, int c1, int cols, int lane, float (&sum)[4])
{
    const uint8_t *rows[N];
#pragma unroll
    for (int j = 0; j < N; j++) rows[j] = x + min(j, last_token) * row_bytes;          // (sums of tokens that are not there are dropped)
    if constexpr (VEC) {
        constexpr int AHEAD = N == 1 ? 4 : 2;
#pragma unroll 1
        for (int c = c0 + lane * 8; c < c1; c += 256 * AHEAD) {
            Eight<DT, true> a[AHEAD], b[AHEAD][N];
#pragma unroll
            for (int u = 0; u < AHEAD; u++) {
                const int at = c + 256 * u < c1 ? c + 256 * u : cols;                  // (columns beyond the end read as zeros)
                a[u] = load_eight<DT, true>(w, at, cols);
#pragma unroll
                for (int j = 0; j < N; j++) b[u][j] = load_eight<DT, true>(rows[j], at, cols);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; u++) {
                float f[8], v[8];
                values_of(a[u], f);
#pragma unroll
                for (int j = 0; j < N; j++) {
                    values_of(b[u][j], v);
#pragma unroll
                    for (int q = 0; q < 8; q++) sum[j] = __fmaf_rn(f[q], v[q], sum[j]);
                }
            }
        }
    } else {
        for (int c = c0 + lane; c < c1; c += 32) {
            const float a = Act<DT>::one(w, c);
#pragma unroll
            for (int j = 0; j < N; j++) sum[j] = __fmaf_rn(a, Act<DT>::one(rows[j], c), sum[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < N; j++)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], o);
}

// logits of this CTA's quarter of the experts, to all four CTAs: an expert and up to four tokens are a task, a warp's or, with few of them,
// shared by `parts` warps, a run of columns each
template <int DT, bool VEC>
__device__ __forceinline__ void router(const MoeFp8 &L, float *logits, float (*partial)[4], uint32_t rank, int warp, int lane)
{
    const int quads = (L.T + 3) / 4, tasks = (L.experts + CLUSTER - 1) / CLUSTER * quads;
    int shift = 0;                                        // parts = 2^shift
    while ((tasks << (shift + 1)) <= WARPS) shift++;
    const int width = ((L.hidden + (1 << shift) - 1 >> shift) + 255) / 256 * 256, part = warp & ((1 << shift) - 1);
    for (int task = warp >> shift; task < tasks; task += WARPS >> shift) {
        const int e = (int)rank + CLUSTER * (task / quads), t0 = task % quads * 4;
        float sum[4] = {};
        if (e < L.experts) {
            const uint8_t *w = reinterpret_cast<const uint8_t *>(L.router) + (long long)e * L.hidden * 2;
            const uint8_t *x = reinterpret_cast<const uint8_t *>(L.x) + (long long)t0 * L.hidden * 2;
            const int c0 = part * width, c1 = min(L.hidden, c0 + width);
            if (L.T == 1) router_products<DT, VEC, 1>(w, x, 0, 0, c0, c1, L.hidden, lane, sum);
            else router_products<DT, VEC, 4>(w, x, 2ll * L.hidden, L.T - 1 - t0, c0, c1, L.hidden, lane, sum);
        }
        if (shift > 0) {                                  // (a single round)
            if (lane == 0) *reinterpret_cast<float4 *>(partial[warp]) = make_float4(sum[0], sum[1], sum[2], sum[3]);
            asm volatile("bar.sync 2, %0;" ::"n"(THREADS) : "memory");
            if (part == 0) {
#pragma unroll
                for (int j = 0; j < 4; j++)
                    for (int q = 1; q < 1 << shift; q++) sum[j] += partial[warp + q][j];
            }
        }
        // lane 4 j + r: token t0 + j to CTA r
        const int j = lane >> 2;
        const float v = j == 0 ? sum[0] : j == 1 ? sum[1] : j == 2 ? sum[2] : sum[3];
        if (part == 0 && e < L.experts && j < 4 && t0 + j < L.T) store_peer(logits + (t0 + j) * L.experts + e, (uint32_t)(lane & 3), v);
    }
    // (warps without a task in that round meet the others all the same)
    if (shift > 0 && (warp >> shift) >= tasks) asm volatile("bar.sync 2, %0;" ::"n"(THREADS) : "memory");
}

// an order of FP32 values as unsigned integers; both zeros are equal
__device__ __forceinline__ uint32_t order_of(float v)
{
    const uint32_t b = __float_as_uint(__fadd_rn(v, 0.f));            // (-0 + 0 = 0)
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// a warp: token t's choices and their weights; EACH: experts of a lane
template <int EACH>
__device__ __forceinline__ void choose_experts(const MoeFp8 &L, const float *logits, int t, int lane, int16_t *chosen, float *weight)
{
    const float *mine = logits + t * L.experts;
    uint32_t key[EACH];                                   // 0: no expert, or chosen already
    float v[EACH], top = -__int_as_float(0x7F800000), total = 0.f;
#pragma unroll
    for (int i = 0; i < EACH; i++) {
        const int e = lane + 32 * i;
        v[i] = e < L.experts ? mine[e] : -__int_as_float(0x7F800000);
        key[i] = e < L.experts ? max(order_of(v[i]), 1u) : 0u;
        top = fmaxf(top, v[i]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
#pragma unroll
    for (int i = 0; i < EACH; i++) total += lane + 32 * i < L.experts ? expf(v[i] - top) : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    int choice = 0;                                       // lane j: choice j
#pragma unroll 1
    for (int j = 0; j < L.top; j++) {
        uint32_t best = key[0];
#pragma unroll
        for (int i = 1; i < EACH; i++) best = max(best, key[i]);
        const uint32_t most = __reduce_max_sync(0xffffffffu, best);
        uint32_t e = 0x7FFFFFFFu;
#pragma unroll
        for (int i = EACH - 1; i >= 0; i--)
            if (key[i] == most) e = (uint32_t)(lane + 32 * i);
        const int winner = (int)__reduce_min_sync(0xffffffffu, e);
#pragma unroll
        for (int i = 0; i < EACH; i++)
            if (winner == lane + 32 * i) key[i] = 0u;
        if (lane == j) choice = winner;
    }
    const float p = lane < L.top ? expf(mine[choice] - top) / total : 0.f;
    float picked = p;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) picked += __shfl_xor_sync(0xffffffffu, picked, o);
    if (lane < L.top) {
        chosen[t * L.top + lane] = (int16_t)choice;
        weight[t * L.top + lane] = L.renormalize ? p / picked : p;
    }
}

// all threads: the entries, experts ascending, an expert's pairs ascending
__device__ __forceinline__ void list_entries(const MoeFp8 &L, const int16_t *chosen, Plan *plan, int *warp_total)
{
    const int e = threadIdx.x, warp = e >> 5, lane = e & 31, pairs = L.T * L.top;
    int count = 0;
    if (e < L.experts)
#pragma unroll 8
        for (int p = 0; p < pairs; p++) count += chosen[p] == e ? 1 : 0;
    const int entries = (count + TOKENS - 1) / TOKENS;
    int before = entries;                                 // inclusive sum over the warp, then over the warps
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int other = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += other;
    }
    if (lane == 31) warp_total[warp] = before;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < WARPS; w++) {
        if (w < warp) before += warp_total[w];
        all += warp_total[w];
    }
    if (threadIdx.x == 0) plan->entries = all;
    int at = before - entries, n = 0;
    if (count > 0)
        for (int p = 0; p < pairs; p++)
            if (chosen[p] == e) {
                plan->pair[at][n] = (int16_t)p;
                if (++n == TOKENS) { plan->expert[at] = (int16_t)e; plan->count[at++] = TOKENS; n = 0; }
            }
    if (n > 0) { plan->expert[at] = (int16_t)e; plan->count[at] = (int16_t)n; }
    __syncthreads();
}

// ---- shared memory: [ring: a stage a warp][two sets of sums][plan][choices][barriers]; the logits lie in the ring until that is used --------
constexpr int UP_STAGE = UP_GROUPS * GROUP_BYTES, UP_STRIDE = UP_GROUPS * GROUP + 4;
constexpr int UP_PART = WARPS * TOKENS * UP_STRIDE * 4;
constexpr int OFF_PART = WARPS * UP_STAGE, OFF_PLAN = OFF_PART + 2 * UP_PART, OFF_CHOSEN = OFF_PLAN + (int)sizeof(Plan),
              OFF_UP_BARS = OFF_CHOSEN + MAX_ENTRIES * 2, UP_SMEM = OFF_UP_BARS + (WARPS + 2) * 8 + WARPS * 4;
static_assert(UP_SMEM + 1024 <= 232448 && MOE_MAX_TOKENS * MOE_MAX_EXPERTS * 4 <= OFF_PART && sizeof(Plan) % 16 == 0, "");

template <int DT, bool VEC>
__global__ void __launch_bounds__(THREADS, 1)
moe_gate_up_kernel(const __grid_constant__ CUtensorMap map_gate, const __grid_constant__ CUtensorMap map_up, const __grid_constant__ Params P)
{
    extern __shared__ __align__(1024) uint8_t sm[];
    __shared__ float peaks[2][TOKENS][CLUSTER];           // largest magnitudes of the four CTAs' columns of h
    const MoeFp8 &L = P.L;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float *logits = reinterpret_cast<float *>(sm), *part = reinterpret_cast<float *>(sm + OFF_PART);
    Plan *plan = reinterpret_cast<Plan *>(sm + OFF_PLAN);
    int16_t *chosen = reinterpret_cast<int16_t *>(sm + OFF_CHOSEN);
    int *warp_total = reinterpret_cast<int *>(sm + OFF_UP_BARS + (WARPS + 2) * 8);
    const uint32_t peak_bars = smem_addr(sm + OFF_UP_BARS) + 8 * WARPS;            // two: the peaks of a pass are complete
    const uint32_t bar = smem_addr(sm + OFF_UP_BARS) + 8 * warp, stage = smem_addr(sm) + warp * UP_STAGE;
    if (lane == 0) {
        mbar_init(bar, 1);
        if (warp < 2) mbar_init(peak_bars + 8 * warp, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    uint32_t rank;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    __syncwarp();
    cluster_sync();                                       // every CTA of the cluster runs: its memory may be written
    pdl_launch_dependents();
    pdl_wait();
    const int kbs = (L.hidden + FP8_BLOCK - 1) / FP8_BLOCK, cluster = (int)blockIdx.x / CLUSTER, clusters = (int)gridDim.x / CLUSTER;
    uint8_t *xq = P.xq + (long long)cluster * L.T * P.xq_pitch;
    float *xs = P.xs + (long long)cluster * L.T * kbs;
    quantize_tokens<DT, VEC>(L, xq, xs, P.xq_pitch, rank);
    router<DT, VEC>(L, logits, reinterpret_cast<float(*)[4]>(part), rank, warp, lane);
    __syncwarp();
    cluster_sync();
    for (int t = warp; t < L.T; t += WARPS) {
        if (L.experts <= 64) choose_experts<2>(L, logits, t, lane, chosen, plan->weight);
        else choose_experts<MOE_MAX_EXPERTS / 32>(L, logits, t, lane, chosen, plan->weight);
    }
    __syncthreads();
    list_entries(L, chosen, plan, warp_total);
    if (blockIdx.x == 0)                                  // for the second kernel
        for (int i = threadIdx.x; i < (int)(sizeof(Plan) / 16); i += THREADS)
            reinterpret_cast<uint4 *>(P.plan)[i] = reinterpret_cast<const uint4 *>(plan)[i];
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");                   // the logits were written where the copies go
    __syncthreads();

    // this cluster's passes: 128 columns of h of an entry each (fewer than 2^25 in all); this CTA's two units of a pass
    const int per_entry = (L.inner + FP8_BLOCK - 1) / FP8_BLOCK;
    const int all = plan->entries * per_entry, share = all / clusters, larger = all - share * clusters, begin = cluster * share + min(cluster, larger);
    const int passes = share + (cluster < larger ? 1 : 0);
    uint32_t gave_up = 0;
    struct Pass { int entry, block, left; };
    auto advance = [&](Pass &p) {
        p.left--;
        if (++p.block == per_entry) { p.block = 0; p.entry++; }
    };
    Pass now = {begin / per_entry, begin % per_entry, passes};
    // the warp's blocks in order: blocks warp, warp + 16, ... of one pass after the other; `ahead` is the one behind the block at work: its
    // tokens and scales are fetched while that is multiplied, its weights as soon as the stage has been read.  (Rows beyond the
    // expert's are read with the boxes and dropped.)
    Pass ahead = now;
    int ahead_kb = warp;
    if (warp >= kbs) ahead.left = 0;
    auto load = [&]() {
        const int row = plan->expert[ahead.entry] * L.inner + ahead.block * FP8_BLOCK + (int)rank * (UNITS * GROUP);
        mbar_expect_tx(bar, UP_STAGE);
        tma_load_2d(stage, &map_gate, ahead_kb * FP8_BLOCK, row, bar);
        tma_load_2d(stage + UP_STAGE / 2, &map_up, ahead_kb * FP8_BLOCK, row, bar);
    };
    const int g = lane >> 2, t = lane & 3;
    TokenRaw<VPTQ_DTYPE_E4M3, true> x;
    float x_scale = 0.f, ws = 0.f;                        // ws: lane 0 the gate's scale of the block, lane 1 the up's
    auto fetch = [&]() {
        const bool any = ahead.left > 0;
        const int entry = any ? ahead.entry : 0;
        const bool mine = any && g < plan->count[entry];
        const int token = mine ? plan->pair[entry][g] / L.top : 0;
        x = load_e4m3(mine ? xq + (long long)token * P.xq_pitch : nullptr, t, ahead_kb, P.xq_pitch);
        x_scale = mine ? __ldcg(xs + token * kbs + ahead_kb) : 0.f;
        ws = any ? __ldg((lane & 1 ? L.up_scale : L.gate_scale) + ((long long)plan->expert[entry] * per_entry + ahead.block) * kbs + ahead_kb) : 0.f;
    };
    auto next_block = [&]() {
        ahead_kb += WARPS;
        if (ahead_kb >= kbs) { ahead_kb = warp; advance(ahead); }
    };
    if (ahead.left > 0 && lane == 0) load();
    fetch();

    const int row = (g >> 1) | ((g & 1) << 2);            // (see linear_fp8_decode.cu)
    const uint32_t at0 = (uint32_t)(row * FP8_BLOCK + ((t ^ row) << 4)), at1 = (uint32_t)(row * FP8_BLOCK + (((t + 4) ^ row) << 4));
    const int iterations = warp < kbs ? (kbs - warp + WARPS - 1) / WARPS : 0;
    uint32_t parity = 0, which = 0, peak_parity = 0;
    for (; now.left > 0; advance(now), peak_parity ^= which, which ^= 1u) {
        float acc[UP_GROUPS][1][4] = {};
#pragma unroll 1
        for (int i = 0; i < iterations; i++) {
            const TokenFrag tokens[1] = {quantize_token<VPTQ_DTYPE_E4M3, true>(x, x_scale)};
            const float2 s = scales_of_columns(tokens[0].scale, t);
            const float w0 = __shfl_sync(0xffffffffu, ws, 0), w1 = __shfl_sync(0xffffffffu, ws, 1);
            next_block();
            fetch();
            mbar_wait_within(bar, parity, P.wait_limit, gave_up);
            parity ^= 1u;
#pragma unroll
            for (int r0 = 0; r0 < UP_GROUPS; r0 += UNITS) {
                WeightFrag a[UNITS];
#pragma unroll
                for (int r = 0; r < UNITS; r++) {
                    const uint32_t box = stage + (r0 + r) * GROUP_BYTES;
                    a[r].q[0][0] = load_shared16(box + at0); a[r].q[1][0] = load_shared16(box + 8 * FP8_BLOCK + at0);
                    a[r].q[0][1] = load_shared16(box + at1); a[r].q[1][1] = load_shared16(box + 8 * FP8_BLOCK + at1);
                }
                const float w = r0 == 0 ? w0 : w1;
                block_products<UNITS, 1>(&acc[r0], a, tokens, [&](int, int) { return make_float2(s.x * w, s.y * w); });
            }
            __syncwarp();                                 // every lane has read the stage
            if (ahead.left > 0 && !__any_sync(0xffffffffu, gave_up != 0) && lane == 0) load();
        }
        // (two sets of sums, and of magnitudes: one is read while the next pass's warps that are done write the other.  A CTA two passes ahead has
        // had this one's magnitudes of the pass between, which leave behind the barrier that every reader of this pass's comes to.)
        float *sums = part + which * (WARPS * TOKENS * UP_STRIDE), *mine = sums + warp * TOKENS * UP_STRIDE;
#pragma unroll
        for (int r = 0; r < UP_GROUPS; r++)
#pragma unroll
            for (int i = 0; i < 4; i++) mine[(2 * t + (i & 1)) * UP_STRIDE + r * GROUP + row + 8 * (i >> 1)] = acc[r][0][i];
        // A wait of any warp that gave up, here or in a pass before, ends this CTA's part: from here on its columns of h are NaN and it sends no
        // magnitudes, so that its peers' waits run out as well.  (One that went on sending would be passes ahead of those that wait for it.)
        const bool lost = __syncthreads_or(gave_up != 0);
        if (lost) gave_up = 1;
        if (threadIdx.x == 0 && !lost) mbar_expect_tx(peak_bars + 8 * which, (uint32_t)plan->count[now.entry] * CLUSTER * 4);
        // a warp a token, a lane a column
        const bool has = warp < plan->count[now.entry];
        const int col = now.block * FP8_BLOCK + (int)rank * (UNITS * GROUP) + lane;
        float h = 0.f;
        if (has) {
            float gate = 0.f, up = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; w++) {
                gate += sums[(w * TOKENS + warp) * UP_STRIDE + lane];
                up += sums[(w * TOKENS + warp) * UP_STRIDE + UNITS * GROUP + lane];
            }
            if (col < L.inner) h = gate / (1.f + expf(-gate)) * up;
            uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(h) & 0x7FFFFFFFu);
            if (!lost) {
                if (lane < CLUSTER) store_peer_async(&peaks[which][warp][rank], peak_bars + 8 * which, (uint32_t)lane, __uint_as_float(most));
                __syncwarp();
                mbar_wait_within(peak_bars + 8 * which, peak_parity, P.wait_limit, gave_up);
            }
            most = 0;
#pragma unroll
            for (int r = 0; r < CLUSTER; r++) most = max(most, __float_as_uint(peaks[which][warp][r]));
            // (its columns and, from rank 0, the block's scale)
            if (__any_sync(0xffffffffu, gave_up != 0)) { h = __int_as_float(0x7FFFFFFF); most = 0x7FFFFFFFu; }
            const Fp8Scale s = fp8_scale(__uint_as_float(most));
            const int pair = plan->pair[now.entry][warp];
            if (col < P.hq_pitch) P.hq[(long long)pair * P.hq_pitch + col] = col < L.inner ? (uint8_t)fp8_pair(h * s.factor, 0.f) : (uint8_t)0;
            if (rank == 0 && lane == 0) P.hs[(long long)pair * per_entry + now.block] = s.scale;
        }
    }
    // A CTA whose waits gave up did not see all of its peers' magnitudes arrive: it stays until all have sent theirs.  (The others have had the
    // last pass's from all four.)
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    if (__any_sync(0xffffffffu, gave_up != 0)) {
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        let_copies_land();
    }
}

// ---- the down projection -----------------------------------------------------------------------------------
// shared memory: [ring: stages][slots: [warp][token][groups * 16 + 4]][plan][barriers]
__host__ __device__ inline int down_slot_floats(int tokens, int groups) { return tokens * (groups * GROUP + 4); }

__global__ void __launch_bounds__(THREADS, 1)
moe_down_kernel(const __grid_constant__ CUtensorMap map_down, const __grid_constant__ Params P, int stages)
{
    extern __shared__ __align__(1024) uint8_t sm[];
    const MoeFp8 &L = P.L;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int block_bytes = P.down_groups * GROUP_BYTES, run_shift = P.down_run_shift, run = 1 << run_shift, stage_bytes = block_bytes << run_shift;
    const int stride = P.down_groups * GROUP + 4;
    float *slots = reinterpret_cast<float *>(sm + (long long)WARPS * stages * stage_bytes), *mine = slots + warp * down_slot_floats(L.T, P.down_groups);
    Plan *plan = reinterpret_cast<Plan *>(slots + WARPS * down_slot_floats(L.T, P.down_groups));
    const uint32_t bars = smem_addr(plan + 1) + (uint32_t)(8 * warp * stages), ring = smem_addr(sm) + (uint32_t)(warp * stages * stage_bytes);
    if (lane == 0) {
        for (int s = 0; s < stages; s++) mbar_init(bars + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_launch_dependents();
    pdl_wait();                                           // the plan and h are the first kernel's
    for (int i = threadIdx.x; i < (int)(sizeof(Plan) / 16); i += THREADS)
        reinterpret_cast<uint4 *>(plan)[i] = __ldcg(reinterpret_cast<const uint4 *>(P.plan) + i);
    __syncthreads();

    const int groups = (L.hidden + GROUP - 1) / GROUP, kbs = (L.inner + FP8_BLOCK - 1) / FP8_BLOCK, runs = (kbs + run - 1) >> run_shift;
    const int first = (int)((long long)groups * blockIdx.x / gridDim.x), count = (int)((long long)groups * (blockIdx.x + 1) / gridDim.x) - first;
    const int pass_groups = count / P.down_passes, larger = count - pass_groups * P.down_passes;
    auto pass_begin = [&](int p) { return first + p * pass_groups + min(p, larger); };
    const int scale_rows = (L.hidden + FP8_BLOCK - 1) / FP8_BLOCK;
    // this warp's loads, in order: runs warp, warp + 16, ... of the entries one after the other, pass by pass
    struct At { int pass, entry, r; };
    auto settle = [&](At &a) {                            // r counts on from the entry before
        while (a.pass < P.down_passes && a.r >= runs) {
            a.r -= runs;
            if (++a.entry == plan->entries) { a.entry = 0; a.pass++; a.r = warp; }
        }
    };
    At ahead = {0, 0, warp};
    settle(ahead);
    uint32_t gave_up = 0;
    auto load = [&](uint32_t slot) {
        const uint32_t bar = bars + 8 * slot, to = ring + slot * stage_bytes;
        const int row = plan->expert[ahead.entry] * L.hidden + pass_begin(ahead.pass) * GROUP;
        mbar_expect_tx(bar, (uint32_t)stage_bytes);
        if (run_shift > 0) tma_load_3d(to, &map_down, 0, row, ahead.r << run_shift, bar);
        else tma_load_2d(to, &map_down, ahead.r * FP8_BLOCK, row, bar);
    };
    for (int s = 0; s < stages && ahead.pass < P.down_passes; s++) {
        if (lane == 0) load((uint32_t)s);
        ahead.r += WARPS;
        settle(ahead);
    }
    __syncwarp();

    const int g = lane >> 2, t = lane & 3;
    const int row = (g >> 1) | ((g & 1) << 2);
    const uint32_t at0 = (uint32_t)(row * FP8_BLOCK + ((t ^ row) << 4)), at1 = (uint32_t)(row * FP8_BLOCK + (((t + 4) ^ row) << 4));
    uint32_t slot = 0, parity = 0;
    // the block at work, and the one behind it, whose h and scales are fetched while that is multiplied
    struct Block { At at; int kb, end; };                 // a block of the run `at`, which ends at `end`
    auto begin_run = [&](Block &b) {
        settle(b.at);
        b.kb = b.at.r << run_shift;
        b.end = min(kbs, b.kb + run);
    };
    auto next_block = [&](Block &b) {
        if (++b.kb == b.end) { b.at.r += WARPS; begin_run(b); }
    };
    Block now = {{0, 0, warp}, 0, 0};
    begin_run(now);
    Block next = now;
    TokenRaw<VPTQ_DTYPE_E4M3, true> x;
    float x_scale = 0.f, ws = 0.f;                        // ws: lanes 0, 1: scales of the pass's two groups in the block
    auto fetch = [&]() {
        const bool any = next.at.pass < P.down_passes;
        const int entry = any ? next.at.entry : 0, group = any ? pass_begin(next.at.pass) + (lane & 1) : 0;
        const bool mine = any && g < plan->count[entry];
        const int pair = mine ? plan->pair[entry][g] : 0;
        x = load_e4m3(mine ? P.hq + (long long)pair * P.hq_pitch : nullptr, t, next.kb, P.hq_pitch);
        x_scale = mine ? __ldcg(P.hs + (long long)pair * kbs + next.kb) : 0.f;
        ws = any ? __ldg(L.down_scale + ((long long)plan->expert[entry] * scale_rows + min(group / (FP8_BLOCK / GROUP), scale_rows - 1)) * kbs + next.kb) : 0.f;
    };
    fetch();
    for (int p = 0; p < P.down_passes; p++) {
        const int g0 = pass_begin(p), n_groups = pass_begin(p + 1) - g0;
        for (int i = lane; i < down_slot_floats(L.T, P.down_groups); i += 32) mine[i] = 0.f;
        __syncwarp();
        float acc[DOWN_GROUPS][1][4] = {};
#pragma unroll 1
        while (now.at.pass == p) {
            const TokenFrag tokens[1] = {quantize_token<VPTQ_DTYPE_E4M3, true>(x, x_scale)};
            const float2 s = scales_of_columns(tokens[0].scale, t);
            const float w0 = __shfl_sync(0xffffffffu, ws, 0), w1 = __shfl_sync(0xffffffffu, ws, 1);
            next_block(next);
            fetch();
            const int in_run = now.kb - (now.at.r << run_shift), entry = now.at.entry;
            if (in_run == 0) mbar_wait_within(bars + 8 * slot, parity, P.wait_limit, gave_up);
            WeightFrag a[DOWN_GROUPS];
#pragma unroll
            for (int r = 0; r < DOWN_GROUPS; r++) {
                // (one group: the other's operands are whatever lies behind, dropped)
                const uint32_t box = ring + slot * stage_bytes + (uint32_t)(in_run * block_bytes + r * GROUP_BYTES);
                a[r].q[0][0] = load_shared16(box + at0); a[r].q[1][0] = load_shared16(box + 8 * FP8_BLOCK + at0);
                a[r].q[0][1] = load_shared16(box + at1); a[r].q[1][1] = load_shared16(box + 8 * FP8_BLOCK + at1);
            }
            block_products<DOWN_GROUPS, 1>(acc, a, tokens, [&](int r, int) { return r == 0 ? make_float2(s.x * w0, s.y * w0) : make_float2(s.x * w1, s.y * w1); });
            if (now.kb == now.end - 1) {
                __syncwarp();                             // every lane has read the stage
                if (ahead.pass < P.down_passes) {
                    if (!__any_sync(0xffffffffu, gave_up != 0) && lane == 0) load(slot);
                    ahead.r += WARPS;
                    settle(ahead);
                }
                if (++slot == (uint32_t)stages) { slot = 0; parity ^= 1u; }
            }
            now = next;
            if (now.at.pass != p || now.at.entry != entry) {
                // the entry's sums; each (row, token) is one lane's: an expert has a token once
                const int n = plan->count[entry];
                const bool lost = __any_sync(0xffffffffu, gave_up != 0);
#pragma unroll
                for (int r = 0; r < DOWN_GROUPS; r++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const int j = 2 * t + (i & 1);
                        if (r < n_groups && j < n) {
                            const int pair = plan->pair[entry][j];
                            float *to = mine + pair / L.top * stride + r * GROUP + row + 8 * (i >> 1);
                            *to = __fmaf_rn(plan->weight[pair], lost ? __int_as_float(0x7FFFFFFF) : acc[r][0][i], *to);
                        }
                        acc[r][0][i] = 0.f;
                    }
                __syncwarp();
            }
        }
        __syncthreads();
        const int rows = n_groups * GROUP, m0 = g0 * GROUP;
        for (int i = threadIdx.x; i < L.T * rows; i += THREADS) {
            const int token = i / rows, m = i % rows;
            if (m0 + m >= L.hidden) continue;
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; w++) sum += slots[w * down_slot_floats(L.T, P.down_groups) + token * stride + m];
            store_out(L.out, (long long)token * L.hidden + m0 + m, sum, L.out_dtype);
        }
        __syncthreads();
    }
    if (gave_up) let_copies_land();
}

// workspace: plan, h and its scales, a copy of x and its scales for every cluster
struct Workspace { long long hq, hs, xq, xs, bytes; };
Workspace workspace_of(int hidden, int inner, int top, int T)
{
    auto up = [](long long v) { return (v + 255) / 256 * 256; };
    const long long clusters = device_sm_count() / CLUSTER > 0 ? device_sm_count() / CLUSTER : 1, pairs = (long long)T * top;
    Workspace w;
    w.hq = up((long long)sizeof(Plan));
    w.hs = up(w.hq + pairs * fp8_row_bytes(inner));
    w.xq = up(w.hs + 4 * pairs * ceil_div(inner, FP8_BLOCK));
    w.xs = up(w.xq + clusters * T * fp8_row_bytes(hidden));
    w.bytes = up(w.xs + 4 * clusters * T * ceil_div(hidden, FP8_BLOCK));
    return w;
}

}  // namespace

long long moe_fp8_workspace_bytes(int hidden, int inner, int top, int T) { return workspace_of(hidden, inner, top, T).bytes; }

cudaError_t launch_moe_fp8(const MoeFp8 &L, void *ws, cudaStream_t st)
{
    const Workspace w = workspace_of(L.hidden, L.inner, L.top, L.T);
    uint8_t *w8 = reinterpret_cast<uint8_t *>(ws);
    Params P;
    P.L = L;
    P.plan = reinterpret_cast<Plan *>(w8);
    P.hq = w8 + w.hq; P.hs = reinterpret_cast<float *>(w8 + w.hs);
    P.xq = w8 + w.xq; P.xs = reinterpret_cast<float *>(w8 + w.xs);
    P.hq_pitch = (int)fp8_row_bytes(L.inner); P.xq_pitch = (int)fp8_row_bytes(L.hidden);
    P.wait_limit = wait_limit();
    const int sms = device_sm_count();
    const long long pitch_h = fp8_row_bytes(L.hidden), pitch_i = fp8_row_bytes(L.inner);
    const int down_all = ceil_div(L.hidden, GROUP), down_grid = down_all < sms ? down_all : sms, most = ceil_div(down_all, down_grid);
    const int down_kbs = ceil_div(L.inner, FP8_BLOCK);
    P.down_passes = ceil_div(most, DOWN_GROUPS);
    P.down_groups = ceil_div(most, P.down_passes);
    P.down_run_shift = 0;
    if (L.inner % FP8_BLOCK == 0 && (long long)down_kbs * L.top >= 2 * WARPS) P.down_run_shift = 1;
    CUtensorMap gate, up, down;
    const long long rows_i = (long long)L.experts * L.inner, rows_h = (long long)L.experts * L.hidden;
    if (!encode_tensor_map(&gate, CU_TENSOR_MAP_DATA_TYPE_UINT8, L.gate, pitch_h, rows_i, pitch_h, 0, 0, FP8_BLOCK, UNITS * GROUP, 1, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !encode_tensor_map(&up, CU_TENSOR_MAP_DATA_TYPE_UINT8, L.up, pitch_h, rows_i, pitch_h, 0, 0, FP8_BLOCK, UNITS * GROUP, 1, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !(P.down_run_shift > 0 ? encode_tensor_map(&down, CU_TENSOR_MAP_DATA_TYPE_UINT8, L.down, FP8_BLOCK, rows_h, pitch_i, down_kbs, FP8_BLOCK, FP8_BLOCK,
                                                   P.down_groups * GROUP, 1 << P.down_run_shift, CU_TENSOR_MAP_SWIZZLE_128B)
                               : encode_tensor_map(&down, CU_TENSOR_MAP_DATA_TYPE_UINT8, L.down, pitch_i, rows_h, pitch_i, 0, 0, FP8_BLOCK, P.down_groups * GROUP, 1,
                                                   CU_TENSOR_MAP_SWIZZLE_128B)))
        return cudaErrorNotSupported;

    const bool vec = L.hidden % 8 == 0;
    auto kern = L.x_dtype == VPTQ_DTYPE_BF16 ? (vec ? moe_gate_up_kernel<VPTQ_DTYPE_BF16, true> : moe_gate_up_kernel<VPTQ_DTYPE_BF16, false>)
                                             : (vec ? moe_gate_up_kernel<VPTQ_DTYPE_FP16, true> : moe_gate_up_kernel<VPTQ_DTYPE_FP16, false>);
    cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void *>(kern), UP_SMEM);
    if (e != cudaSuccess) return e;
    int clusters = max_resident_clusters(reinterpret_cast<const void *>(kern), CLUSTER, THREADS, UP_SMEM);
    if (clusters < 1) return cudaErrorNotSupported;
    if (clusters > sms / CLUSTER && sms >= CLUSTER) clusters = sms / CLUSTER;      // (the workspace has no more copies)
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(CLUSTER * clusters));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = UP_SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CLUSTER; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = pdl_enabled("moe_fp8") ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, kern, gate, up, P);
    if (e != cudaSuccess) return e;

    const int stage = P.down_groups * GROUP_BYTES << P.down_run_shift;
    const int fixed = WARPS * down_slot_floats(L.T, P.down_groups) * 4 + (int)sizeof(Plan) + WARPS * 8 * 8;
    int stages = (232448 - fixed) / (WARPS * stage);
    if (stages > 8) stages = 8;
    const int smem = stages * WARPS * stage + fixed;
    e = allow_dynamic_smem(reinterpret_cast<const void *>(moe_down_kernel), 232448);
    if (e != cudaSuccess) return e;
    cfg.gridDim = dim3((unsigned)down_grid);
    cfg.dynamicSmemBytes = smem;
    cfg.attrs = attr + 1; cfg.numAttrs = pdl_enabled("moe_fp8") ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, moe_down_kernel, down, P, stages);
}

}  // namespace vptq
