// Tiled tensor maps of matrices and the loads through them (no multicast).
#pragma once
#include <cuda.h>

#include "common.cuh"

namespace vptq {

// map of a row-major matrix: `cols` values of `type` a row, rows `row_bytes` apart (a multiple of 16), boxes of box_rows x box_cols;
// `layers` > 0: a third dimension of matrices `layer_bytes` apart, boxes box_layers deep (device_info.cu)
bool encode_tensor_map(CUtensorMap *map, CUtensorMapDataType type, const void *p, uint64_t cols, uint64_t rows, uint64_t row_bytes, uint64_t layers,
                       uint64_t layer_bytes, uint32_t box_cols, uint32_t box_rows, uint32_t box_layers, CUtensorMapSwizzle swizzle);

#ifdef __CUDACC__
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// a map on its way to where the first copy through it needs it
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
#endif

}  // namespace vptq
