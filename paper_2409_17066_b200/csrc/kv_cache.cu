// Keys and values of tokens into the pages of a quantized cache, and out of them.
//
// A row (token, keys or values, head) is dealt with in pieces of 128 columns by 8 lanes, sixteen adjacent columns each (rows of at most 64
// columns by 4 lanes): 32 bytes of 16-bit values, 16 (e4m3) or 8 bytes (e2m1) of codes.  Its scale is one shuffle (e2m1) or three
// (e4m3), by the rules of the matrices (fp8.cuh, fp4.cuh).
// A CTA takes some tokens: a thread looks up the place of each (a binary search for its sequence, then its page) and leaves it in shared
// memory, and every thread goes through its tokens with one and the same piece of a row, so that what changes from token to token is three
// addresses.  Up to four tokens' reads are in flight a thread; when writing, the first four before the places are known.
// Nothing outside the cache is touched whatever the tables say: tokens without a sequence, positions beyond the table and pages that the
// cache does not have are not written; read, they give zeros (tokens without a sequence: nothing).
// Bound by HBM where there are many tokens, by the latency of dependent reads (sequences, start, page, codes) where there are few.
#include "kv_cache.cuh"

namespace vptq {

namespace {

constexpr int THREADS = 256;

struct CacheParams {
    KvCache C;
    int row_bytes, scale_bytes;                // of a row in the cache
    int chunks, units;                         // pieces of a row, and of a token (keys and values of all heads)
    int width, groups;                         // pieces of a token that a CTA takes, and tokens that it takes side by side
    int wide;                                  // rows to be read lie on 32 bytes, in pieces of 32 bytes
};

// Where a token's rows of head 0 begin, in bytes of codes and in bytes of scales; negative: GONE, it has no page, or NONE, it is in no sequence.
constexpr long long GONE = -1, NONE = -2;
struct __align__(16) Place { long long codes, scales; };

__device__ __forceinline__ Place find_place(const CacheParams &P, int t)
{
    const KvCache &C = P.C;
    int lo = 0, n = C.seqs;                    // the last sequence that does not begin behind t is in [lo, lo + n)
    while (n > 1) {
        const int half = n / 2;
        if (__ldg(C.cu + lo + half) <= t) { lo += half; n -= half; }
        else n = half;
    }
    const int begin = __ldg(C.cu + lo), end = __ldg(C.cu + lo + 1), start = __ldg(C.start + lo);
    if (t < begin || t >= end) return {NONE, NONE};
    const long long token = (long long)start + ((long long)t - begin);
    if (token < 0 || token > 0xFFFFFFFFll) return {GONE, GONE};    // (a list that begins below zero may ask for more)
    const uint32_t slot = (uint32_t)token / (uint32_t)C.page;
    if (slot >= (uint32_t)C.width) return {GONE, GONE};
    const int page = __ldg(C.table + (long long)lo * C.width + slot);
    if ((unsigned)page >= (unsigned)C.pages) return {GONE, GONE};
    const long long row = (long long)page * C.heads * C.page + ((uint32_t)token - slot * (uint32_t)C.page);
    return {row * P.row_bytes, row * P.scale_bytes};
}

// What a thread works on: keys or values, a head, its first column of sixteen, and the tokens first, first + groups, ... of the CTA's.
struct Piece { int kv, head, c, first; bool any; };
template <int LANES>
__device__ __forceinline__ Piece piece_of(const CacheParams &P)
{
    const int slot = threadIdx.x / LANES, group = slot / P.width, unit = blockIdx.y * P.width + slot - group * P.width;
    const int row = unit / P.chunks, kv = row >= P.C.heads ? 1 : 0;
    return {kv, row - kv * P.C.heads, (unit - row * P.chunks) * FP8_BLOCK + (int)(threadIdx.x % LANES) * 16, group, group < P.groups && unit < P.units};
}

constexpr int BATCH = 4;                       // tokens of a thread whose reads are in flight together

// e4m3 codes of sixteen values, of which the first `n` exist (the others are zeros, whatever the factor)
template <int DT, bool VEC>
__device__ __forceinline__ uint4 e4m3_codes16(const Sixteen<DT, VEC> &e, float f, int n)
{
    uint32_t w[4];
#pragma unroll
    for (int h = 0; h < 2; h++) {
        float v[8], t[8];
        values_of(e.h[h], v);
#pragma unroll
        for (int i = 0; i < 8; i += 2) times2(t[i], t[i + 1], v[i], v[i + 1], f);
        w[2 * h] = fp8_quad(t[0], t[1], t[2], t[3]);
        w[2 * h + 1] = fp8_quad(t[4], t[5], t[6], t[7]);
    }
    if (n < 16)
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = n >= 4 * i + 4 ? w[i] : n <= 4 * i ? 0u : w[i] & ((1u << (8 * (n - 4 * i))) - 1u);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// the places of a CTA's tokens, the first of them t0
__device__ __forceinline__ void find_places(const CacheParams &P, int t0, int tokens, Place *place)
{
    for (int i = threadIdx.x; i < tokens; i += THREADS) place[i] = t0 + i < P.C.tokens ? find_place(P, t0 + i) : Place{NONE, NONE};
    __syncthreads();
}

// N tokens a thread
template <int DT, bool VEC, bool E2M1, int LANES, int N>
__global__ void __launch_bounds__(THREADS)
cache_write_kernel(const __grid_constant__ CacheParams P)
{
    constexpr int TOGETHER = N < BATCH ? N : BATCH;
    __shared__ Place place[THREADS / LANES / 2 * N];
    const KvCache &C = P.C;
    pdl_wait();
    const int tokens = N * P.groups, t0 = (int)blockIdx.x * tokens, lane = threadIdx.x % LANES;
    const Piece p = piece_of<LANES>(P);
    const long long step = P.groups * C.token_stride[p.kv] * Act<DT>::BYTES;
    const uint8_t *x = reinterpret_cast<const uint8_t *>(C.x[p.kv]) + ((t0 + p.first) * C.token_stride[p.kv] + p.head * C.head_stride[p.kv]) * Act<DT>::BYTES;
    const long long head_rows = (long long)p.head * C.page;
    uint8_t *q = C.q[p.kv] + head_rows * P.row_bytes + (E2M1 ? p.c / 2 : p.c);
    uint8_t *scale = reinterpret_cast<uint8_t *>(C.scale[p.kv]) + head_rows * P.scale_bytes + (E2M1 ? p.c / FP4_BLOCK : p.c / FP8_BLOCK * 4);
    const bool in_row = (E2M1 ? p.c / 2 : p.c) < P.row_bytes;
#pragma unroll 1
    for (int k = 0; k < N; k += TOGETHER) {
        Sixteen<DT, VEC> e[TOGETHER];
#pragma unroll
        for (int i = 0; i < TOGETHER; i++) {
            const int t = p.first + (k + i) * P.groups;
            e[i] = load_sixteen<DT, VEC>(x, p.any && t0 + t < C.tokens ? p.c : C.dim, C.dim);
            x += step;
        }
        if (k == 0) find_places(P, t0, tokens, place);
#pragma unroll
        for (int i = 0; i < TOGETHER; i++) {
            uint32_t m = magnitude(e[i]);
            const Place at = p.any ? place[p.first + (k + i) * P.groups] : Place{NONE, NONE};
            if constexpr (E2M1) {
                const uint32_t b = fp4_pair_scale(m);
                if (at.codes < 0 || !in_row) continue;
                *reinterpret_cast<uint2 *>(q + at.codes) = fp4_codes16(e[i], b, C.dim - p.c);
                if ((lane & 1) == 0) scale[at.scales] = (uint8_t)b;
            } else {
#pragma unroll
                for (int o = LANES / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
                if (at.codes < 0) continue;
                const Fp8Scale s = fp8_scale(__uint_as_float(m));
                if (in_row) *reinterpret_cast<uint4 *>(q + at.codes) = e4m3_codes16(e[i], s.factor, C.dim - p.c);
                if (lane == 0) *reinterpret_cast<float *>(scale + at.scales) = s.scale;
            }
        }
    }
}

__device__ __forceinline__ void e4m3_scaled8(uint2 q, float s, float (&v)[8])
{
    uint32_t h[4];
    asm("{\n\t.reg .b16 a, b, c, d;\n\tmov.b32 {a, b}, %4;\n\tmov.b32 {c, d}, %5;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\tcvt.rn.f16x2.e4m3x2 %2, c;\n\tcvt.rn.f16x2.e4m3x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(q.x), "r"(q.y));
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[i]));
        times2(v[2 * i], v[2 * i + 1], f.x, f.y, s);
    }
}

template <int DT, bool VEC, bool E2M1, int LANES, int N>
__global__ void __launch_bounds__(THREADS)
cache_read_kernel(const __grid_constant__ CacheParams P)
{
    constexpr int TOGETHER = N < BATCH ? N : BATCH, BYTES = DT == VPTQ_DTYPE_FP32 ? 4 : 2;
    __shared__ Place place[THREADS / LANES / 2 * N];
    const KvCache &C = P.C;
    pdl_wait();
    const int tokens = N * P.groups, t0 = (int)blockIdx.x * tokens;
    const Piece p = piece_of<LANES>(P);
    const long long step = P.groups * C.token_stride[p.kv] * BYTES;
    uint8_t *x = reinterpret_cast<uint8_t *>(C.x[p.kv]) + ((t0 + p.first) * C.token_stride[p.kv] + p.head * C.head_stride[p.kv]) * BYTES;
    const long long head_rows = (long long)p.head * C.page;
    const uint8_t *q = C.q[p.kv] + head_rows * P.row_bytes + (E2M1 ? p.c / 2 : p.c);
    const uint8_t *scale = reinterpret_cast<const uint8_t *>(C.scale[p.kv]) + head_rows * P.scale_bytes + (E2M1 ? p.c / FP4_BLOCK : p.c / FP8_BLOCK * 4);
    find_places(P, t0, tokens, place);
    if (!p.any || p.c >= C.dim) return;
#pragma unroll 1
    for (int k = 0; k < N; k += TOGETHER) {
        uint4 codes[TOGETHER];
        float s[TOGETHER];
        bool in[TOGETHER];
#pragma unroll
        for (int i = 0; i < TOGETHER; i++) {
            const Place at = place[p.first + (k + i) * P.groups];
            in[i] = at.codes != NONE;
            codes[i] = make_uint4(0, 0, 0, 0);
            s[i] = 0.f;
            if (at.codes < 0) continue;
            if constexpr (E2M1) {
                const uint2 w = __ldcs(reinterpret_cast<const uint2 *>(q + at.codes));
                codes[i].x = w.x; codes[i].y = w.y;
                s[i] = fp4_scale_value(__ldg(scale + at.scales));
            } else {
                codes[i] = __ldcs(reinterpret_cast<const uint4 *>(q + at.codes));
                s[i] = __ldg(reinterpret_cast<const float *>(scale + at.scales));
            }
        }
#pragma unroll
        for (int i = 0; i < TOGETHER; i++) {
            float lo[8], hi[8];
            if constexpr (E2M1) {
                fp4_scaled8(codes[i].x, s[i], lo);
                fp4_scaled8(codes[i].y, s[i], hi);
            } else {
                e4m3_scaled8(make_uint2(codes[i].x, codes[i].y), s[i], lo);
                e4m3_scaled8(make_uint2(codes[i].z, codes[i].w), s[i], hi);
            }
            if (in[i]) store_values16<DT, VEC>(x, p.c, C.dim, P.wide, lo, hi);
            x += step;
        }
    }
}

template <int DT, bool VEC, bool E2M1, int LANES, bool WRITE, int N>
cudaError_t launch(const CacheParams &P, int parts, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ceil_div(P.C.tokens, N * P.groups), (unsigned)parts);
    cfg.blockDim = dim3(THREADS);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled("kv_cache") ? 1 : 0;
    if constexpr (WRITE) return cudaLaunchKernelEx(&cfg, cache_write_kernel<DT, VEC, E2M1, LANES, N>, P);
    else return cudaLaunchKernelEx(&cfg, cache_read_kernel<DT, VEC, E2M1, LANES, N>, P);
}

// Pieces of a token are dealt out evenly to CTAs of THREADS / LANES slots; what is left of the slots takes more tokens.  A thread takes one, four or
// sixteen tokens: the more, the fewer look-ups and addresses, but the more registers (CTAs that an SM holds: reading 8, 4 or 5, 3 or 4; writing 6, 4, 3;
// writing out of FP32 6, 2, 2) and the fewer threads.  The steps are by the CTAs of the one-token form, in units of eight an SM.  Measured over heads of
// 40 to 256 columns, the time of the next form over that of the one before:
//   reading, four tokens:              0.5 units 1.1, 1 0.9 to 1.0, 2 0.84, 8 0.8 to 0.9, 96 0.7 to 0.9
//   reading, sixteen instead of four:  2 1.2 to 1.6, 8 0.94 to 1.24, 16 0.98 to 1.08, 48 0.95 to 1.05, 96 0.90 to 1.02
//   writing, four:                     0.5 1.0 to 1.2, 1 0.9 to 1.0, 2 0.9, 8 0.8, 96 0.7; sixteen instead of four: 1.0 to 1.2 from 8 on, not taken
//   writing out of FP32, four:         1.1 to 1.2 from 1 on, not taken; sixteen instead of one: 8 1.0, 24 1.0, 48 1.0, 64 0.9, 96 0.9
template <int DT, bool VEC, bool E2M1, int LANES, bool WRITE>
cudaError_t launch_tokens(CacheParams P, cudaStream_t st)
{
    constexpr int SLOTS = THREADS / LANES;
    const int parts = ceil_div(P.units, SLOTS);
    P.width = ceil_div(P.units, parts);
    P.groups = SLOTS / P.width;
    const long long ctas = (long long)ceil_div(P.C.tokens, P.groups) * parts, unit = (long long)device_sm_count() * 8;
    if constexpr (!(WRITE && DT == VPTQ_DTYPE_FP32)) {
        if (ctas > unit && (WRITE || ctas < 48 * unit)) return launch<DT, VEC, E2M1, LANES, WRITE, 4>(P, parts, st);
    }
    if constexpr (!(WRITE && DT != VPTQ_DTYPE_FP32)) {
        if (ctas >= 48 * unit) return launch<DT, VEC, E2M1, LANES, WRITE, 16>(P, parts, st);
    }
    return launch<DT, VEC, E2M1, LANES, WRITE, 1>(P, parts, st);
}

template <int DT, bool VEC, bool WRITE>
cudaError_t launch_form(const CacheParams &P, cudaStream_t st)
{
    if (P.C.e2m1) return P.C.dim <= 64 ? launch_tokens<DT, VEC, true, 4, WRITE>(P, st) : launch_tokens<DT, VEC, true, 8, WRITE>(P, st);
    return P.C.dim <= 64 ? launch_tokens<DT, VEC, false, 4, WRITE>(P, st) : launch_tokens<DT, VEC, false, 8, WRITE>(P, st);
}

template <bool WRITE>
cudaError_t launch_cache(const KvCache &C, cudaStream_t st)
{
    CacheParams P;
    P.C = C;
    P.row_bytes = (int)(C.e2m1 ? fp4_row_bytes(C.dim) : fp8_row_bytes(C.dim));
    P.scale_bytes = C.e2m1 ? ceil_div(C.dim, FP4_BLOCK) : 4 * ceil_div(C.dim, FP8_BLOCK);
    P.chunks = ceil_div(C.dim, FP8_BLOCK);
    P.units = 2 * C.heads * P.chunks;
    P.width = P.groups = 0;
    const int bytes = C.x_dtype == VPTQ_DTYPE_FP32 ? 4 : 2, per = 16 / bytes;
    bool vec = C.dim % per == 0;
    P.wide = C.dim % 16 == 0 && ((reinterpret_cast<uintptr_t>(C.x[0]) | reinterpret_cast<uintptr_t>(C.x[1])) & 31u) == 0;      // (read: packed)
    for (int i = 0; i < 2; i++)
        vec = vec && (reinterpret_cast<uintptr_t>(C.x[i]) & 15u) == 0 && (C.tokens == 1 || C.token_stride[i] % per == 0) && (C.heads == 1 || C.head_stride[i] % per == 0);
    switch (C.x_dtype) {
    case VPTQ_DTYPE_FP16: return vec ? launch_form<VPTQ_DTYPE_FP16, true, WRITE>(P, st) : launch_form<VPTQ_DTYPE_FP16, false, WRITE>(P, st);
    case VPTQ_DTYPE_BF16: return vec ? launch_form<VPTQ_DTYPE_BF16, true, WRITE>(P, st) : launch_form<VPTQ_DTYPE_BF16, false, WRITE>(P, st);
    default: return vec ? launch_form<VPTQ_DTYPE_FP32, true, WRITE>(P, st) : launch_form<VPTQ_DTYPE_FP32, false, WRITE>(P, st);
    }
}

}  // namespace

cudaError_t launch_cache_write(const KvCache &C, cudaStream_t st) { return launch_cache<true>(C, st); }
cudaError_t launch_cache_read(const KvCache &C, cudaStream_t st) { return launch_cache<false>(C, st); }

}  // namespace vptq
