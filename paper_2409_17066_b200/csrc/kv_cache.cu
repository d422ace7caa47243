// Keys and values of tokens into the pages of a quantized cache, and out of them.
//
// A row (token, keys or values, head) is dealt with in pieces of 128 columns by 16 lanes, eight adjacent columns each (rows of at most 64
// columns by 8 lanes): a 16-byte load of 16-bit values, 8 (e4m3) or 4 bytes (e2m1) of codes.  Its scale is two shuffles (e2m1) or four
// (e4m3), by the rules of the matrices (fp8.cuh, fp4.cuh).
// All pieces of a warp belong to one token, whose place every warp looks up for itself: the token's sequence by a search of 32 places at a
// time (two rounds for 1024 sequences), then its page.  When writing, the values are on their way to the registers meanwhile.
// Nothing outside the cache is touched whatever the tables say: tokens without a sequence, positions beyond the table and pages that the
// cache does not have are not written; read, they give zeros (tokens without a sequence: nothing).
// Bound by HBM where there are many tokens, by the latency of three dependent reads (sequences, start, page) where there are few.
#include "kv_cache.cuh"

namespace vptq {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;

struct CacheParams {
    KvCache C;
    long long row_bytes, scales;               // of a row in the cache
    int chunks, units;                         // pieces of a row, and of a token (keys and values of all heads)
    int warps;                                 // warps that share a token
};

// Place of token t: the cache row of head 0, -1 when it has none, -2 when it is in no sequence.  For a whole warp.
__device__ __forceinline__ long long find_row(const KvCache &C, int t)
{
    // the last sequence that does not begin behind t (the first entry of a group of `stride` that its lanes look at stands for all)
    const int lane = threadIdx.x & 31;
    int lo = 0, n = C.seqs;
    while (true) {
        const int stride = (n + 31) / 32, i = lane * stride;
        const bool before = i < n && __ldg(C.cu + lo + i) <= t;
        const int count = __popc(__ballot_sync(0xffffffffu, before));
        if (count == 0) return -2;
        lo += (count - 1) * stride;
        if (stride == 1) break;
        n = min(stride, n - (count - 1) * stride);
    }
    const int begin = __ldg(C.cu + lo), end = __ldg(C.cu + lo + 1), start = __ldg(C.start + lo);
    if (t < begin || t >= end) return -2;
    const long long token = (long long)start + (t - begin);
    const long long slot = token / C.page;
    if (token < 0 || slot >= C.width) return -1;
    const int page = __ldg(C.table + (long long)lo * C.width + slot);
    if ((unsigned)page >= (unsigned)C.pages) return -1;
    return (long long)page * C.heads * C.page + token % C.page;
}

// Piece `unit` of a token: which of keys and values, which head, which columns.
struct Piece { int kv, head, c; };
__device__ __forceinline__ Piece piece_of(const CacheParams &P, int unit, int c0)
{
    const int row = unit / P.chunks, kv = row >= P.C.heads ? 1 : 0;
    return {kv, row - kv * P.C.heads, (unit - row * P.chunks) * FP8_BLOCK + c0};
}

template <int DT, bool VEC, bool E2M1, int LANES, int ROUNDS>
__global__ void __launch_bounds__(THREADS)
cache_write_kernel(const __grid_constant__ CacheParams P)
{
    constexpr int PER_WARP = 32 / LANES;
    const KvCache &C = P.C;
    pdl_wait();
    const long long w = (long long)blockIdx.x * WARPS + (threadIdx.x >> 5);
    const int t = (int)(w / P.warps), lane = threadIdx.x & (LANES - 1);
    if (t >= C.tokens) return;
    const int unit0 = (int)(w % P.warps) * ROUNDS * PER_WARP + (int)(threadIdx.x & 31) / LANES;
    Eight<DT, VEC> e[ROUNDS];
#pragma unroll
    for (int i = 0; i < ROUNDS; i++) {
        const int unit = unit0 + i * PER_WARP;
        const Piece p = piece_of(P, unit < P.units ? unit : 0, lane * 8);
        const long long at = t * C.token_stride[p.kv] + p.head * C.head_stride[p.kv];
        e[i] = load_eight<DT, VEC>(reinterpret_cast<const uint8_t *>(C.x[p.kv]) + at * Act<DT>::BYTES, unit < P.units ? p.c : C.dim, C.dim);
    }
    const long long row0 = find_row(C, t);
    if (row0 < 0) return;
#pragma unroll
    for (int i = 0; i < ROUNDS; i++) {
        const int unit = unit0 + i * PER_WARP;
        const Piece p = piece_of(P, unit < P.units ? unit : 0, lane * 8);
        const long long row = row0 + (long long)p.head * C.page;
        uint32_t m = magnitude(e[i]);
        if constexpr (E2M1) {
            const uint32_t b = fp4_block_scale(m);
            if (unit >= P.units || p.c / 2 >= P.row_bytes) continue;
            float v[8];
            values_of(e[i], v);
            *reinterpret_cast<uint32_t *>(C.q[p.kv] + row * P.row_bytes + p.c / 2) = fp4_codes(v, b, C.dim - p.c);
            if ((lane & 3) == 0) reinterpret_cast<uint8_t *>(C.scale[p.kv])[row * P.scales + p.c / FP4_BLOCK] = (uint8_t)b;
        } else {
#pragma unroll
            for (int o = LANES / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
            if (unit >= P.units) continue;
            const Fp8Scale s = fp8_scale(__uint_as_float(m));
            store_eight(C.q[p.kv] + row * P.row_bytes, P.row_bytes, p.c, C.dim, e[i], s.factor);
            if (lane == 0) reinterpret_cast<float *>(C.scale[p.kv])[row * P.scales + p.c / FP8_BLOCK] = s.scale;
        }
    }
}

__device__ __forceinline__ void e4m3_values8(uint2 q, float (&v)[8])
{
    uint32_t h[4];
    asm("{\n\t.reg .b16 a, b, c, d;\n\tmov.b32 {a, b}, %4;\n\tmov.b32 {c, d}, %5;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\tcvt.rn.f16x2.e4m3x2 %2, c;\n\tcvt.rn.f16x2.e4m3x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(q.x), "r"(q.y));
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[i]));
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
}

template <int DT, bool VEC, bool E2M1, int LANES, int ROUNDS>
__global__ void __launch_bounds__(THREADS)
cache_read_kernel(const __grid_constant__ CacheParams P)
{
    constexpr int PER_WARP = 32 / LANES;
    const KvCache &C = P.C;
    pdl_wait();
    const long long w = (long long)blockIdx.x * WARPS + (threadIdx.x >> 5);
    const int t = (int)(w / P.warps), lane = threadIdx.x & (LANES - 1);
    if (t >= C.tokens) return;
    const int unit0 = (int)(w % P.warps) * ROUNDS * PER_WARP + (int)(threadIdx.x & 31) / LANES;
    const long long row0 = find_row(C, t);
    if (row0 == -2) return;
    uint2 q[ROUNDS];
    float s[ROUNDS];
#pragma unroll
    for (int i = 0; i < ROUNDS; i++) {
        const int unit = unit0 + i * PER_WARP;
        q[i] = make_uint2(0, 0);
        s[i] = 0.f;
        if (row0 < 0 || unit >= P.units) continue;
        const Piece p = piece_of(P, unit, lane * 8);
        if (p.c >= C.dim) continue;
        const long long row = row0 + (long long)p.head * C.page;
        if constexpr (E2M1) {
            q[i].x = __ldcs(reinterpret_cast<const uint32_t *>(C.q[p.kv] + row * P.row_bytes + p.c / 2));
            s[i] = fp4_scale_value(__ldg(reinterpret_cast<const uint8_t *>(C.scale[p.kv]) + row * P.scales + p.c / FP4_BLOCK));
        } else {
            q[i] = __ldcs(reinterpret_cast<const uint2 *>(C.q[p.kv] + row * P.row_bytes + p.c));
            s[i] = __ldg(reinterpret_cast<const float *>(C.scale[p.kv]) + row * P.scales + p.c / FP8_BLOCK);
        }
    }
#pragma unroll
    for (int i = 0; i < ROUNDS; i++) {
        const int unit = unit0 + i * PER_WARP;
        if (unit >= P.units) break;
        const Piece p = piece_of(P, unit, lane * 8);
        float v[8];
        if constexpr (E2M1) fp4_values8(q[i].x, v);
        else e4m3_values8(q[i], v);
#pragma unroll
        for (int k = 0; k < 8; k++) v[k] *= s[i];
        const long long at = t * C.token_stride[p.kv] + p.head * C.head_stride[p.kv];
        store_values8<DT, VEC>(reinterpret_cast<uint8_t *>(C.x[p.kv]) + at * (DT == VPTQ_DTYPE_FP32 ? 4 : 2), p.c, C.dim, v);
    }
}

template <int DT, bool VEC, bool E2M1, int LANES, int ROUNDS>
cudaError_t launch(CacheParams P, bool write, cudaStream_t st)
{
    P.warps = ceil_div(P.units, 32 / LANES * ROUNDS);
    const long long ctas = ((long long)P.C.tokens * P.warps + WARPS - 1) / WARPS;
    if (write) return launch_dependent("cache_write", cache_write_kernel<DT, VEC, E2M1, LANES, ROUNDS>, (int)ctas, THREADS, 0, st, P);
    return launch_dependent("cache_read", cache_read_kernel<DT, VEC, E2M1, LANES, ROUNDS>, (int)ctas, THREADS, 0, st, P);
}

// few pieces: one to 8 or 16 lanes; more than fill the device twice over: four, so that the search for the token's place serves as many
template <int DT, bool VEC, bool E2M1, int LANES>
cudaError_t launch_rounds(const CacheParams &P, bool write, cudaStream_t st)
{
    const long long warps = (long long)P.C.tokens * ceil_div(P.units, 32 / LANES);
    if (warps <= (long long)device_sm_count() * 128) return launch<DT, VEC, E2M1, LANES, 1>(P, write, st);
    return launch<DT, VEC, E2M1, LANES, 4>(P, write, st);
}

template <int DT, bool VEC>
cudaError_t launch_form(const CacheParams &P, bool write, cudaStream_t st)
{
    if (P.C.e2m1) return P.C.dim <= 64 ? launch_rounds<DT, VEC, true, 8>(P, write, st) : launch_rounds<DT, VEC, true, 16>(P, write, st);
    return P.C.dim <= 64 ? launch_rounds<DT, VEC, false, 8>(P, write, st) : launch_rounds<DT, VEC, false, 16>(P, write, st);
}

cudaError_t launch_cache(const KvCache &C, bool write, cudaStream_t st)
{
    CacheParams P;
    P.C = C;
    P.row_bytes = C.e2m1 ? fp4_row_bytes(C.dim) : fp8_row_bytes(C.dim);
    P.scales = ceil_div(C.dim, C.e2m1 ? FP4_BLOCK : FP8_BLOCK);
    P.chunks = ceil_div(C.dim, FP8_BLOCK);
    P.units = 2 * C.heads * P.chunks;
    P.warps = 0;
    const int bytes = C.x_dtype == VPTQ_DTYPE_FP32 ? 4 : 2, per = 16 / bytes;
    bool vec = C.dim % per == 0;
    for (int i = 0; i < 2; i++)
        vec = vec && (reinterpret_cast<uintptr_t>(C.x[i]) & 15u) == 0 && (C.tokens == 1 || C.token_stride[i] % per == 0) && (C.heads == 1 || C.head_stride[i] % per == 0);
    switch (C.x_dtype) {
    case VPTQ_DTYPE_FP16: return vec ? launch_form<VPTQ_DTYPE_FP16, true>(P, write, st) : launch_form<VPTQ_DTYPE_FP16, false>(P, write, st);
    case VPTQ_DTYPE_BF16: return vec ? launch_form<VPTQ_DTYPE_BF16, true>(P, write, st) : launch_form<VPTQ_DTYPE_BF16, false>(P, write, st);
    default: return vec ? launch_form<VPTQ_DTYPE_FP32, true>(P, write, st) : launch_form<VPTQ_DTYPE_FP32, false>(P, write, st);
    }
}

}  // namespace

cudaError_t launch_cache_write(const KvCache &C, cudaStream_t st) { return launch_cache(C, true, st); }
cudaError_t launch_cache_read(const KvCache &C, cudaStream_t st) { return launch_cache(C, false, st); }

}  // namespace vptq
