// A vector-quantized layer restored straight to an e4m3 weight with 128 x 128 block scales: the FP16 values of vptq_dequant, bit for
// bit (FP32, three separately rounded operations, then FP16), quantized by the rule of fp8_quantize.cu, without the FP16 matrix in
// global memory.
//
// A CTA makes a 128 x 128 block at a time and leaves its FP16 values in shared memory; the block's maximum and the rounding follow.
// A thread takes four adjacent columns of a vector row: their indices are one window of packed words, their values leave as 8-byte
// stores (one column to a thread: 8192 x 28672 with 65536 + 256 entries 322 us instead of 254; eight to a thread spill: 335). Columns that do not lie so, under
// a permutation, beside the outliers, at other index widths, are looked up one to a thread, ITEMS vector rows at a time so that as many
// table reads are in flight.
// A vector row that crosses a block's edge is looked up by both blocks (v = 8 never does; v = 6: 23 rows instead of 21.3).
// TABLES: main and residual table of a layer with one group are staged in shared memory as 16-byte rows, and two CTAs an SM go through
// the blocks; out of L1 every 4-byte piece of a 12-byte row is a wavefront of its own for each lane (11008 x 4096 with v = 6: 97 us
// instead of 75).  Blocks are dealt out column of blocks by column, so that those with outliers, which take twice as long, come first and to
// CTAs of their own (row by row some CTAs had three of them: 75 us instead of 62).
// A table in L2 (1 MiB) makes a random read a vector, one a clock and SM; what it takes beyond them are dependent reads, indices and then
// rows, with one block at a time a CTA (4096 x 4096 17.8 us, of which the reads are 8).  A small table is bound by the arithmetic (8192 x 28672
// with 256 entries 201 us).
// E2M1: the same to e2m1 with a power of two for every 32 columns of a row (fp4.cuh), for layers that the kernel of dequant_fp4.cu does not take:
// only what follows the FP16 values differs.
#include "fp4.cuh"
#include "index_words.cuh"
#include "restore_words.cuh"

namespace vptq {

namespace {

// threads of a CTA, and pairs that a thread looks up at a time: out of L2 more CTAs, out of shared memory more threads to hide their
// arithmetic behind one another's (one column to a thread: 8192 x 28672 314 us, 512 threads 367; 11008 x 4096, v = 6, 81, 256 threads 108)
template <bool TABLES> constexpr int threads() { return TABLES ? 512 : 256; }
template <bool TABLES> constexpr int items() { return TABLES ? 2 : 4; }
constexpr int CPL = 4;                                   // adjacent columns that a thread restores together
constexpr int TILE_STRIDE = FP8_BLOCK + 8;                // halves; 16-byte rows, half warps read them without conflicts

struct DequantFp8Params {
    LayerView L;
    uint8_t *q;
    float *scale;             // e4m3
    uint8_t *tiles;           // e2m1: its scales
    const int *inverse;       // stored column of every input feature (-1: none names it), or null
    long long pitch;
    int row_blocks, col_blocks, blocks;
};
constexpr int TABLES_MAX = (115712 - 1024 - FP8_BLOCK * TILE_STRIDE * 2) / 16;         // entries of both tables, two CTAs an SM

// component j of a table row: out of its words, or (V = 0: any length) out of the table
template <int V>
__device__ __forceinline__ float component(const RowWords<V> &r, const __half *__restrict__ tab, long long e, int v, int j)
{
    if constexpr (V > 0) {
        const uint32_t w = r.w[j / 2];
        return __half2float(__ushort_as_half((unsigned short)((j & 1) ? w >> 16 : w & 0xFFFFu)));
    } else {
        return __half2float(__ldg(tab + e * v + j));
    }
}

__device__ __forceinline__ float finish(float t, bool has_scale, float s, float b)
{
    return has_scale ? __fadd_rn(__fmul_rn(t, s), b) : t;              // never contracted to an FMA
}

template <int V, bool TABLES, bool E2M1>
__device__ __forceinline__ void restore_block(const DequantFp8Params &P, int index, __half (*tile)[TILE_STRIDE], uint32_t *part, const uint4 *tables)
{
    constexpr int THREADS = threads<TABLES>(), ITEMS = items<TABLES>();
    constexpr int COL_LANES = THREADS / FP8_BLOCK;        // vector rows of a block taken at a time
    const LayerView &L = P.L;
    const int rb = index % P.row_blocks, cb = index / P.row_blocks;
    const int m0 = rb * FP8_BLOCK, m1 = min(L.M, m0 + FP8_BLOCK);
    const int v = V > 0 ? V : L.v;
    // columns [fast0, fast1) of the block are restored several adjacent ones to a thread, the others one to a thread
    int fast0 = 0, fast1 = 0;
    if constexpr (V > 0) {
        const int b1 = L.s1.bits, b2 = L.k2 > 0 ? L.s2.bits : 8;
        if (P.inverse == nullptr && !L.scale_rows && (b1 == 8 || b1 == 12 || b1 == 16) && (b2 == 8 || b2 == 12 || b2 == 16)) {
            fast0 = min(FP8_BLOCK, (max(0, L.n_out - cb * FP8_BLOCK) + CPL - 1) / CPL * CPL);
            fast1 = min(FP8_BLOCK, (L.N - cb * FP8_BLOCK) / CPL * CPL);
        }
        const int c = (threadIdx.x & 31) * CPL, n = cb * FP8_BLOCK + c, col = n - L.n_out, r1 = (m1 + V - 1) / V;
        const bool res = L.k2 > 0;
        const unsigned bit1 = (unsigned)col * (unsigned)b1, bit2 = (unsigned)col * (unsigned)b2;
        // scale and bias of the columns; without them t * 1 + (-0) = t, whatever t and its sign
        float sc[CPL], bi[CPL];
#pragma unroll
        for (int k = 0; k < CPL; k += 2) {
            float2 fs = make_float2(1.f, 1.f), fb = make_float2(-0.f, -0.f);
            if (L.has_scale && c >= fast0 && c < fast1) {
                fs = __half22float2(__ldg(reinterpret_cast<const __half2 *>(L.scale + n + k)));
                fb = __half22float2(__ldg(reinterpret_cast<const __half2 *>(L.bias + n + k)));
            }
            sc[k] = fs.x; sc[k + 1] = fs.y; bi[k] = fb.x; bi[k + 1] = fb.y;
        }
        for (int r = c >= fast0 && c < fast1 ? m0 / V + (int)(threadIdx.x >> 5) : r1; r < r1; r += THREADS / 32) {
            const IndexWindow<CPL> q1 = load_window<CPL>(L.s1.ptr + (long long)r * L.s1.stride, bit1, (unsigned)(L.s1.stride >> 2));
            IndexWindow<CPL> q2 = {};
            if (res) q2 = load_window<CPL>(L.s2.ptr + (long long)r * L.s2.stride, bit2, (unsigned)(L.s2.stride >> 2));
            int i1[CPL], i2[CPL];
            decode_window<CPL>(q1, bit1 & 31u, b1, L.k1, i1);
            decode_window<CPL>(q2, bit2 & 31u, b2, res ? L.k2 : 1, i2);
            RowWords<V> w1[CPL], w2[CPL];
#pragma unroll
            for (int k = 0; k < CPL; k++) {
                if constexpr (TABLES) {
                    const uint4 a = tables[i1[k]], b = tables[res ? L.k1 + i2[k] : 0];
                    const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                    for (int j = 0; j < V / 2; j++) { w1[k].w[j] = wa[j]; w2[k].w[j] = wb[j]; }
                } else {
                    const long long group = L.G > 1 ? (col + k) / L.cpg : 0;
                    w1[k] = row_from_global<V>(L.c1, group * L.k1 + i1[k]);
                    if (res) w2[k] = row_from_global<V>(L.c2, group * L.k2 + i2[k]);
                }
            }
            const int at = r * V - m0;
            __half *dst = &tile[0][c] + at * TILE_STRIDE;
#pragma unroll
            for (int j = 0; j < V / 2; j++) {
                float2 y[CPL];                                            // components 2j, 2j + 1 of the thread's columns
#pragma unroll
                for (int k = 0; k < CPL; k++) {
                    y[k] = __half22float2(*reinterpret_cast<const __half2 *>(&w1[k].w[j]));
                    if (res) y[k] = add_half2(y[k], w2[k].w[j]);
                    y[k].x = __fadd_rn(__fmul_rn(y[k].x, sc[k]), bi[k]);
                    y[k].y = __fadd_rn(__fmul_rn(y[k].y, sc[k]), bi[k]);
                }
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    __align__(8) __half2 o[CPL / 2];
#pragma unroll
                    for (int k = 0; k < CPL; k += 2) o[k / 2] = __floats2half2_rn(h ? y[k].y : y[k].x, h ? y[k + 1].y : y[k + 1].x);
                    if ((unsigned)(at + 2 * j + h) < (unsigned)(m1 - m0))
                        *reinterpret_cast<uint2 *>(dst + (2 * j + h) * TILE_STRIDE) = *reinterpret_cast<const uint2 *>(o);
                }
            }
        }
    }
    if (fast0 > 0 || fast1 < FP8_BLOCK) {
        const int c = threadIdx.x % FP8_BLOCK, sub = threadIdx.x / FP8_BLOCK;
        const int f = cb * FP8_BLOCK + c;                                 // input feature
        const bool done = c >= fast0 && c < fast1;
        const int n = f >= L.N ? -1 : P.inverse ? __ldg(P.inverse + f) : f;      // stored column
        float sc = 1.f, bi = -0.f;                                        // without them t * 1 + (-0) = t, whatever t and its sign
        if (n >= 0 && L.has_scale && !L.scale_rows) { sc = __half2float(__ldg(L.scale + n)); bi = __half2float(__ldg(L.bias + n)); }
        auto put = [&](int m, float t) {
            float s = sc, b = bi;
            if (L.has_scale && L.scale_rows) { s = __half2float(__ldg(L.scale + m)); b = __half2float(__ldg(L.bias + m)); }
            tile[m - m0][c] = __float2half_rn(finish(t, L.has_scale, s, b));
        };
        if (done) {
        } else if (n < 0) {
            for (int m = m0 + sub; m < m1; m += COL_LANES) tile[m - m0][c] = __float2half_rn(0.f);
        } else if (n < L.n_out) {
            // (few columns, but a wait for every read of each would hold up the whole block: eight indices, then their rows)
            const int r1 = (m1 + L.v0 - 1) / L.v0;
            for (int r0 = m0 / L.v0 + sub; r0 < r1; r0 += COL_LANES * 8) {
                int i0[8];
#pragma unroll
                for (int i = 0; i < 8; i++)
                    i0[i] = clamp_index(load_index(L.s0.ptr + (long long)min(r0 + i * COL_LANES, r1 - 1) * L.s0.stride, n, L.s0.bits), L.k0);
                for (int j = 0; j < L.v0; j++) {
                    float t[8];
#pragma unroll
                    for (int i = 0; i < 8; i++) t[i] = __half2float(__ldg(L.c0 + (long long)i0[i] * L.v0 + j));
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const int r = r0 + i * COL_LANES, m = r * L.v0 + j;
                        if (r < r1 && m >= m0 && m < m1) put(m, t[i]);
                    }
                }
            }
        } else {
            const int col = n - L.n_out, group = L.G > 1 ? col / L.cpg : 0;
            const bool res = L.k2 > 0;
            const int r1 = (m1 + v - 1) / v;                              // (m1 <= M: rows that exist)
            for (int r0 = m0 / v + sub; r0 < r1; r0 += COL_LANES * ITEMS) {
                long long e1[ITEMS], e2[ITEMS];
                RowWords<V> w1[ITEMS], w2[ITEMS];
#pragma unroll
                for (int i = 0; i < ITEMS; i++) {
                    const int r = min(r0 + i * COL_LANES, r1 - 1);
                    e1[i] = (long long)group * L.k1 + clamp_index(load_index(L.s1.ptr + (long long)r * L.s1.stride, col, L.s1.bits), L.k1);
                    e2[i] = res ? (long long)group * L.k2 + clamp_index(load_index(L.s2.ptr + (long long)r * L.s2.stride, col, L.s2.bits), L.k2) : 0;
                }
#pragma unroll
                for (int i = 0; i < ITEMS; i++) {
                    if constexpr (TABLES) {
                        const uint4 q = tables[e1[i]], p = tables[res ? L.k1 + e2[i] : 0];
                        const uint32_t a[4] = {q.x, q.y, q.z, q.w}, b[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
                        for (int k = 0; k < V / 2; k++) { w1[i].w[k] = a[k]; w2[i].w[k] = b[k]; }
                    } else if constexpr (V > 0) {
                        w1[i] = row_from_global<V>(L.c1, e1[i]);
                        if (res) w2[i] = row_from_global<V>(L.c2, e2[i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < ITEMS; i++) {
                    const int r = r0 + i * COL_LANES;
                    if (r >= r1) break;
                    auto one = [&](int j) {
                        const int m = r * v + j;
                        if (m < m0 || m >= m1) return;
                        float t = component<V>(w1[i], L.c1, e1[i], v, j);
                        if (res) t = __fadd_rn(t, component<V>(w2[i], L.c2, e2[i], v, j));
                        put(m, t);
                    };
                    if constexpr (V > 0) {
#pragma unroll
                        for (int j = 0; j < V; j++) one(j);
                    } else {
                        for (int j = 0; j < v; j++) one(j);
                    }
                }
            }
        }
    }
    __syncthreads();
    if constexpr (E2M1) {
        // 8 lanes a row, sixteen columns a lane, two lanes a block (eight columns a lane: 8192 x 8192 with v = 12 103 us instead of 97); the
        // scales of 128 x 128 values are one tile, whose rows beyond M hold zeros
        constexpr int ROWS = THREADS / 8;
        const int lane = threadIdx.x >> 1 & 7, c = cb * FP8_BLOCK + lane * 16;       // (adjacent lanes in adjacent rows: in different banks)
        uint8_t *scales = P.tiles + ((long long)rb * P.col_blocks + cb) * FP4_TILE_BYTES;
#pragma unroll
        for (int i = 0; i < FP8_BLOCK / ROWS; i++) {
            const int row = i * ROWS + (int)(threadIdx.x >> 4 << 1 | (threadIdx.x & 1));
            const bool in = m0 + row < m1;
            Sixteen<VPTQ_DTYPE_FP16, true> e;
#pragma unroll
            for (int h = 0; h < 2; h++) e.h[h].q = in && c < L.N ? *reinterpret_cast<const uint4 *>(&tile[row][lane * 16 + 8 * h]) : make_uint4(0, 0, 0, 0);
            const uint32_t b = fp4_pair_scale<2>(magnitude(e));
            if (in && c / 2 < P.pitch) *reinterpret_cast<uint2 *>(P.q + (long long)(m0 + row) * P.pitch + c / 2) = fp4_codes16(e, b, L.N - c);
            if ((lane & 1) == 0) scales[fp4_scale_at(row, lane >> 1)] = (uint8_t)b;
        }
        return;
    }
    // 16 lanes a row, eight columns a lane (rows beyond M were not written: left out)
    constexpr int ROWS = THREADS / 16, ROUNDS = FP8_BLOCK / ROWS;
    const int lane = threadIdx.x & 15, sub = threadIdx.x >> 4, c = cb * FP8_BLOCK + lane * 8;
    uint4 w[ROUNDS];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < ROUNDS; i++) {
        const int row = i * ROWS + sub;
        w[i] = m0 + row < m1 ? *reinterpret_cast<const uint4 *>(&tile[row][lane * 8]) : make_uint4(0, 0, 0, 0);
        most = __vmaxu2(most, __vmaxu2(__vmaxu2(w[i].x & 0x7FFF7FFFu, w[i].y & 0x7FFF7FFFu), __vmaxu2(w[i].z & 0x7FFF7FFFu, w[i].w & 0x7FFF7FFFu)));
    }
    most = __reduce_max_sync(0xffffffffu, max(most & 0xFFFFu, most >> 16));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 32; i++) most = max(most, part[i]);
    const Fp8Scale s = fp8_scale(__half2float(__ushort_as_half((unsigned short)most)));
    if (threadIdx.x == 0) P.scale[(long long)rb * P.col_blocks + cb] = s.scale;
    if (c >= P.pitch) return;
#pragma unroll
    for (int i = 0; i < ROUNDS; i++) {
        const int row = i * ROWS + sub;
        if (m0 + row >= m1) break;
        const uint32_t h[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
        uint32_t o[2];
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const float2 a = Act<VPTQ_DTYPE_FP16>::two(h[2 * k]), b = Act<VPTQ_DTYPE_FP16>::two(h[2 * k + 1]);
            o[k] = fp8_quad(a.x * s.factor, a.y * s.factor, b.x * s.factor, b.y * s.factor);
        }
        uint8_t *dst = P.q + (long long)(m0 + row) * P.pitch + c;
        *reinterpret_cast<uint2 *>(dst) = make_uint2(o[0], o[1]);
        if (c + 8 > L.N)
            for (int j = max(0, L.N - c); j < 8; j++) dst[j] = 0;         // pad bytes are zeros, whatever the factor
    }
}

template <int V, bool TABLES, bool E2M1>
__global__ void __launch_bounds__(threads<TABLES>(), TABLES ? 2 : V > 8 ? 3 : 4)
dequant_fp8_kernel(const __grid_constant__ DequantFp8Params P)
{
    constexpr int THREADS = threads<TABLES>();
    __shared__ __align__(16) __half tile[FP8_BLOCK][TILE_STRIDE];
    __shared__ uint32_t part[THREADS / 32];
    extern __shared__ __align__(16) uint4 tables[];
    if constexpr (TABLES) {
        for (int i = threadIdx.x; i < P.L.k1 + P.L.k2; i += THREADS)
            tables[i] = i < P.L.k1 ? load_centroid_row(P.L.c1, i, V) : load_centroid_row(P.L.c2, i - P.L.k1, V);
        __syncthreads();
        // (the first blocks may hold outliers, and take longer: the blocks left over for the last round go to other CTAs)
        const int rounds = P.blocks / (int)gridDim.x;
        for (int i = 0; i <= rounds; i++) {
            const int b = i * (int)gridDim.x + (int)(i < rounds ? blockIdx.x : gridDim.x - 1 - blockIdx.x);
            if (b >= P.blocks) break;
            restore_block<V, true, E2M1>(P, b, tile, part, tables);
            __syncthreads();
        }
    } else {
        restore_block<V, false, E2M1>(P, blockIdx.x, tile, part, nullptr);
    }
}

template <int V, bool E2M1>
cudaError_t restore(const DequantFp8Params &P, cudaStream_t st)
{
    if constexpr (V == 6 || V == 8) {
        // staging pays when a CTA reads more rows out of the tables than they have
        const int grid = 2 * device_sm_count(), entries = P.L.k1 + P.L.k2;
        if (P.L.G == 1 && P.L.Nc > 0 && entries <= TABLES_MAX && (long long)P.L.R * P.L.Nc / grid > entries) {
            auto kern = dequant_fp8_kernel<V, true, E2M1>;
            const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void *>(kern), 16ull * TABLES_MAX);
            if (e != cudaSuccess) return e;
            kern<<<P.blocks < grid ? P.blocks : grid, threads<true>(), 16ull * entries, st>>>(P);
            return cudaGetLastError();
        }
    }
    dequant_fp8_kernel<V, false, E2M1><<<P.blocks, threads<false>(), 0, st>>>(P);
    return cudaGetLastError();
}

// stored column order -> the stored column of every feature; a list that is no permutation: the largest column that names it, -1 none
__global__ void __launch_bounds__(256)
inverse_order_kernel(LayerView L, int *inverse)
{
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j < L.N) atomicMax(inverse + in_col(L, j), j);
}

template <bool E2M1>
cudaError_t launch(DequantFp8Params &P, int *inverse, cudaStream_t st)
{
    const LayerView &L = P.L;
    P.inverse = nullptr;
    P.col_blocks = ceil_div(L.N, FP8_BLOCK);
    if (L.perm != nullptr) {
        cudaError_t e = cudaMemsetAsync(inverse, 0xFF, 4ull * L.N, st);
        if (e != cudaSuccess) return e;
        inverse_order_kernel<<<ceil_div(L.N, 256), 256, 0, st>>>(L, inverse);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
        P.inverse = inverse;
    }
    P.row_blocks = ceil_div(L.M, FP8_BLOCK);
    P.blocks = (int)((long long)P.row_blocks * P.col_blocks);
    switch (L.v) {
    case 8: return restore<8, E2M1>(P, st);
    case 6: return restore<6, E2M1>(P, st);
    case 12: return restore<12, E2M1>(P, st);
    default: return restore<0, E2M1>(P, st);
    }
}

}  // namespace

cudaError_t launch_dequant_fp8(const LayerView &L, uint8_t *q, float *scale, int *inverse, cudaStream_t st)
{
    DequantFp8Params P;
    P.L = L; P.q = q; P.scale = scale; P.tiles = nullptr;
    P.pitch = fp8_row_bytes(L.N);
    return launch<false>(P, inverse, st);
}

cudaError_t launch_dequant_fp4(const LayerView &L, uint8_t *q, uint8_t *scale, int *inverse, cudaStream_t st)
{
    if (dequant_fp4_takes(L)) return launch_dequant_fp4_rows(L, q, scale, st);
    static_assert(FP4_TILE_ROWS == FP8_BLOCK && FP4_TILE_COLS == FP8_BLOCK, "a CTA's block is a tile of scales");
    DequantFp8Params P;
    P.L = L; P.q = q; P.scale = nullptr; P.tiles = scale;
    P.pitch = fp4_row_bytes(L.N);
    return launch<true>(P, inverse, st);
}

}  // namespace vptq
