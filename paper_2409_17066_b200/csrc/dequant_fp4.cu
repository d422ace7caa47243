// A vector-quantized layer restored to e2m1, a vector row of 128 columns to a warp: the FP16 values of vptq_dequant, bit for bit, quantized by
// the rule of fp4_quantize.cu.
//
// A lane takes four adjacent columns: their indices are one window of packed words, read for the next piece while this one is quantized, their
// values leave as 8-byte stores to V rows of shared memory that are the warp's own.  Then eight lanes make a row's codes, sixteen columns each, two
// lanes a block.  No warp waits for another, and no vector row is looked up twice, as in the kernel of dequant_fp8.cu, whose CTAs make blocks of
// 128 x 128 (28672 x 8192 with 65536 + 256 entries 252 us, 219 this way; 8192 x 8192 with 256 + 256 entries 70, 56; 11008 x 4096 with v = 6 and
// outliers 59, 54).
// Bound by L1 and shared memory, busy 76 % (a row out of L2, and a random row of a staged table, are a wavefront or more for every lane), and with both
// tables staged by instructions, issue slots 70 % busy.  Rows out of L2 asked for one piece ahead were slower, in spilled registers (295 us).
#include "fp4.cuh"
#include "index_words.cuh"
#include "restore_words.cuh"

namespace vptq {

namespace {

constexpr int CPL = 4, COLS = 32 * CPL;                   // adjacent columns of a lane, and of a warp
constexpr int STRIDE = COLS + 8;                          // halves; 16-byte rows
static_assert(COLS == FP4_TILE_COLS, "a warp's columns are a tile of scales");

constexpr int WARPS = 16, THREADS = 32 * WARPS, CTAS = 2;
template <int V> constexpr int tiles_bytes() { return WARPS * V * STRIDE * 2; }
constexpr int SMEM_MAX = 115712 - 1024;                   // two CTAs an SM

struct Params {
    LayerView L;
    uint8_t *q, *tiles;
    long long pitch;
    int col_blocks, units, scale_rows;     // pieces of a vector row by 128 columns; M rounded up to whole tiles of scales
};

// Shared memory: the warps' rows, then tables as 16-byte rows: BOTH, or the residual's alone.
template <int V, bool BOTH>
__global__ void __launch_bounds__(THREADS, CTAS)
dequant_fp4_kernel(const __grid_constant__ Params P)
{
    extern __shared__ __align__(16) uint4 sm[];
    const LayerView &L = P.L;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool res = L.k2 > 0;
    __half *tile = reinterpret_cast<__half *>(sm) + warp * V * STRIDE;
    uint4 *tables = sm + tiles_bytes<V>() / 16;
    const int n1 = BOTH ? L.k1 : 0;
    const uint4 *table2 = res ? tables + n1 : tables;     // (no residual: a row that is there, and is not added)
    for (int i = threadIdx.x; i < n1 + L.k2; i += THREADS) tables[i] = i < n1 ? load_centroid_row(L.c1, i, V) : load_centroid_row(L.c2, i - n1, V);
    __syncthreads();
    const int b1 = L.s1.bits, b2 = res ? L.s2.bits : 8;
    const int fast0 = (L.n_out + CPL - 1) / CPL * CPL;    // columns from here on, but for the last N % 4, are looked up four to a lane
    const int all = (int)gridDim.x * WARPS, mine = (int)blockIdx.x * WARPS + warp, rounds = P.units / all;
    // (the first pieces may hold outliers, and take longer: those left over for the last round go to other warps)
    auto unit_of = [&](int i) { return i * all + (i < rounds ? mine : all - 1 - mine); };
    struct Where { int r, cb, n; bool some, fast; };
    auto where = [&](int i) {
        const int u = unit_of(i);
        Where w;
        w.cb = u / L.R; w.r = u - w.cb * L.R; w.n = w.cb * COLS + lane * CPL;
        w.some = i <= rounds && u < P.units;
        w.fast = w.some && w.n >= fast0 && w.n + CPL <= L.N;
        return w;
    };
    IndexWindow<CPL> q1 = {}, q2 = {};
    auto load = [&](const Where &w) {
        if (!w.fast) return;
        const unsigned col = (unsigned)(w.n - L.n_out);
        q1 = load_window<CPL>(L.s1.ptr + (long long)w.r * L.s1.stride, col * (unsigned)b1, (unsigned)(L.s1.stride >> 2));
        if (res) q2 = load_window<CPL>(L.s2.ptr + (long long)w.r * L.s2.stride, col * (unsigned)b2, (unsigned)(L.s2.stride >> 2));
    };
    Where w = where(0);
    load(w);
    for (int i = 0; w.some; i++) {
        const int r = w.r, n = w.n, c = lane * CPL;
        if (w.fast) {
            const int col = n - L.n_out;
            int i1[CPL], i2[CPL];
            decode_window<CPL>(q1, (unsigned)col * (unsigned)b1 & 31u, b1, L.k1, i1);
            decode_window<CPL>(q2, (unsigned)col * (unsigned)b2 & 31u, b2, res ? L.k2 : 1, i2);
            RowWords<V> w1[CPL], w2[CPL];
#pragma unroll
            for (int k = 0; k < CPL; k++) {
                if constexpr (BOTH) {
                    const uint4 a = tables[i1[k]];
                    const uint32_t v[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                    for (int j = 0; j < V / 2; j++) w1[k].w[j] = v[j];
                } else {
                    w1[k] = row_from_global<V>(L.c1, i1[k]);
                }
                const uint4 a = table2[i2[k]];
                const uint32_t v[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                for (int j = 0; j < V / 2; j++) w2[k].w[j] = v[j];
            }
            // scale and bias of the columns; without them t * 1 + (-0) = t, whatever t and its sign
            float sc[CPL], bi[CPL];
#pragma unroll
            for (int k = 0; k < CPL; k += 2) {
                float2 fs = make_float2(1.f, 1.f), fb = make_float2(-0.f, -0.f);
                if (L.has_scale) {
                    fs = __half22float2(__ldg(reinterpret_cast<const __half2 *>(L.scale + n + k)));
                    fb = __half22float2(__ldg(reinterpret_cast<const __half2 *>(L.bias + n + k)));
                }
                sc[k] = fs.x; sc[k + 1] = fs.y; bi[k] = fb.x; bi[k + 1] = fb.y;
            }
#pragma unroll
            for (int j = 0; j < V / 2; j++) {
                float2 y[CPL];                                // components 2j, 2j + 1 of the lane's columns
#pragma unroll
                for (int k = 0; k < CPL; k++) {
                    y[k] = __half22float2(*reinterpret_cast<const __half2 *>(&w1[k].w[j]));
                    if (res) y[k] = add_half2(y[k], w2[k].w[j]);
                    y[k].x = __fadd_rn(__fmul_rn(y[k].x, sc[k]), bi[k]);          // (three roundings, never contracted)
                    y[k].y = __fadd_rn(__fmul_rn(y[k].y, sc[k]), bi[k]);
                }
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    __align__(8) __half2 o[CPL / 2];
#pragma unroll
                    for (int k = 0; k < CPL; k += 2) o[k / 2] = __floats2half2_rn(h ? y[k].y : y[k].x, h ? y[k + 1].y : y[k + 1].x);
                    *reinterpret_cast<uint2 *>(tile + (2 * j + h) * STRIDE + c) = *reinterpret_cast<const uint2 *>(o);
                }
            }
        } else {
            // outliers, columns beside them, the last ones and what lies beyond: one at a time
#pragma unroll 1
            for (int k = 0; k < CPL; k++) {
                const int f = n + k;
                float t[V];
#pragma unroll
                for (int j = 0; j < V; j++) t[j] = 0.f;
                if (f < L.n_out) {
#pragma unroll
                    for (int j = 0; j < V; j++) {
                        const int m = min(r * V + j, L.M - 1), r0 = m / L.v0;
                        const int e = clamp_index(load_index(L.s0.ptr + (long long)r0 * L.s0.stride, f, L.s0.bits), L.k0);
                        t[j] = __half2float(__ldg(L.c0 + (long long)e * L.v0 + (m - r0 * L.v0)));
                    }
                } else if (f < L.N) {
                    const int col = f - L.n_out;
                    const long long e1 = clamp_index(load_index(L.s1.ptr + (long long)r * L.s1.stride, col, b1), L.k1);
                    const long long e2 = res ? clamp_index(load_index(L.s2.ptr + (long long)r * L.s2.stride, col, b2), L.k2) : 0;
#pragma unroll
                    for (int j = 0; j < V; j++) {
                        t[j] = __half2float(__ldg(L.c1 + e1 * V + j));
                        if (res) t[j] = __fadd_rn(t[j], __half2float(__ldg(L.c2 + e2 * V + j)));
                    }
                }
                if (f < L.N && L.has_scale) {
                    const float s = __half2float(__ldg(L.scale + f)), b = __half2float(__ldg(L.bias + f));
#pragma unroll
                    for (int j = 0; j < V; j++) t[j] = __fadd_rn(__fmul_rn(t[j], s), b);
                }
#pragma unroll
                for (int j = 0; j < V; j++) tile[j * STRIDE + c + k] = __float2half_rn(t[j]);
            }
        }
        const Where next = where(i + 1);
        load(next);
        __syncwarp();
        const int cb = w.cb, piece = lane >> 1 & 7, first = cb * COLS + piece * 16;
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const int row = j + (lane & 1) + 2 * (lane >> 4), m = r * V + row;
            const bool in = (V % 4 == 0 || row < V) && m < L.M;
            Sixteen<VPTQ_DTYPE_FP16, true> e;
#pragma unroll
            for (int h = 0; h < 2; h++) e.h[h].q = in ? *reinterpret_cast<const uint4 *>(tile + row * STRIDE + piece * 16 + 8 * h) : make_uint4(0, 0, 0, 0);
            const uint32_t b = fp4_pair_scale<2>(magnitude(e));
            if (in && first / 2 < P.pitch) *reinterpret_cast<uint2 *>(P.q + (long long)m * P.pitch + first / 2) = fp4_codes16(e, b, L.N - first);
            if (in && (lane & 2) == 0)
                P.tiles[((long long)(m / FP4_TILE_ROWS) * P.col_blocks + cb) * FP4_TILE_BYTES + fp4_scale_at(m % FP4_TILE_ROWS, piece >> 1)] = (uint8_t)b;
        }
        // rows that the last tile of scales has and the matrix has not
        if (r == L.R - 1)
            for (int m = L.M + (lane >> 2); m < P.scale_rows; m += 8)
                P.tiles[((long long)(m / FP4_TILE_ROWS) * P.col_blocks + cb) * FP4_TILE_BYTES + fp4_scale_at(m % FP4_TILE_ROWS, lane & 3)] = 0;
        __syncwarp();
        w = next;
    }
}

template <int V, bool BOTH>
cudaError_t run(const Params &P, cudaStream_t st)
{
    auto kern = dequant_fp4_kernel<V, BOTH>;
    const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void *>(kern), SMEM_MAX);
    if (e != cudaSuccess) return e;
    const int most = ceil_div(P.units, WARPS), grid = CTAS * device_sm_count();
    kern<<<most < grid ? most : grid, THREADS, tiles_bytes<V>() + 16 * ((BOTH ? P.L.k1 : 0) + P.L.k2), st>>>(P);
    return cudaGetLastError();
}

bool narrow(int bits) { return bits == 8 || bits == 12 || bits == 16; }

// What a CTA stages: 2 both tables, 1 the residual's, 0 neither.  Staging pays when a CTA reads more rows out of the tables than they have.
int staged(const LayerView &L)
{
    const long long read = (long long)L.R * L.Nc / (CTAS * device_sm_count()), most = (SMEM_MAX - (L.v == 6 ? tiles_bytes<6>() : tiles_bytes<8>())) / 16;
    if (L.k1 + L.k2 <= most && read > L.k1 + L.k2) return 2;
    return L.k2 > 0 && L.k2 <= most && read > L.k2 ? 1 : 0;
}

}  // namespace

// Without a table in shared memory the kernel of dequant_fp8.cu, whose CTAs share a block, is faster (11008 x 4096 with 65536 entries 42 us, 47 this way).
bool dequant_fp4_takes(const LayerView &L)
{
    return (L.v == 6 || L.v == 8) && L.perm == nullptr && !L.scale_rows && L.G == 1 && L.Nc > 0 && narrow(L.s1.bits) && (L.k2 == 0 || narrow(L.s2.bits)) &&
           (long long)L.R * ceil_div(L.N, COLS) < 1ll << 30 && staged(L) > 0;
}

cudaError_t launch_dequant_fp4_rows(const LayerView &L, uint8_t *q, uint8_t *scale, cudaStream_t st)
{
    Params P;
    P.L = L; P.q = q; P.tiles = scale;
    P.pitch = fp4_row_bytes(L.N);
    P.col_blocks = ceil_div(L.N, COLS);
    P.units = L.R * P.col_blocks;
    P.scale_rows = ceil_div(L.M, FP4_TILE_ROWS) * FP4_TILE_ROWS;
    const bool both = staged(L) == 2;
    if (L.v == 6) return both ? run<6, true>(P, st) : run<6, false>(P, st);
    return both ? run<8, true>(P, st) : run<8, false>(P, st);
}

}  // namespace vptq
