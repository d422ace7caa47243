// Keys and values in pages, in e4m3 or e2m1 (kv_cache.cu).
#pragma once
#include "fp4.cuh"

namespace vptq {

struct KvCache {
    int heads, dim, page, pages;               // tokens of a page, pages of the cache
    int seqs, width, tokens;                   // sequences, table entries of each, tokens of the call
    int e2m1, x_dtype;
    uint8_t *q[2];                             // keys, values: [pages][heads][page][row bytes]
    void *scale[2];                            // [pages][heads][page][blocks of a row]
    const int *table, *start, *cu;
    void *x[2];                                // [tokens][heads][dim], read or written
    long long token_stride[2], head_stride[2]; // in values
};

cudaError_t launch_cache_write(const KvCache &C, cudaStream_t st);
cudaError_t launch_cache_read(const KvCache &C, cudaStream_t st);

}  // namespace vptq
