// A mixture-of-experts layer for a few tokens (moe_fp8.cu).
#pragma once
#include "fp8.cuh"

namespace vptq {

constexpr int MOE_MAX_TOKENS = VPTQ_MOE_MAX_TOKENS, MOE_MAX_EXPERTS = VPTQ_MOE_MAX_EXPERTS, MOE_MAX_TOP = VPTQ_MOE_MAX_TOP;

struct MoeFp8 {
    int hidden, inner, experts, top, T;
    int x_dtype, out_dtype, renormalize;
    const void *x, *router;                               // [T][hidden], [experts][hidden] of x_dtype
    const uint8_t *gate, *up, *down;                      // [experts][inner][row(hidden)] twice, [experts][hidden][row(inner)]
    const float *gate_scale, *up_scale, *down_scale;
    void *out;                                            // [T][hidden]
};

long long moe_fp8_workspace_bytes(int hidden, int inner, int top, int T);
cudaError_t launch_moe_fp8(const MoeFp8 &L, void *ws, cudaStream_t st);

}  // namespace vptq
