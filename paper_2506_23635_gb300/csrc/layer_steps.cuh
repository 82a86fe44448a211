// The layer's own steps (moe_api.cu), for the layer over 8-bit experts (quant.cu): what dims
// and a token count have to be, the router with its logits, routing and dispatch in as few
// launches as the size allows, the dispatch, the combine.
#pragma once

#include "moe_internal.cuh"

namespace moe {

moe_status check_layer_dims(const moe_dims *d);
moe_status check_layer_tokens(const moe_dims *d, int32_t T);
cudaError_t launch_layer_route(const moe_dims &d, int T, const void *x, const void *w_router,
                               float *logits, int32_t *idx, float *gate, cudaStream_t st);
cudaError_t launch_layer_route_dispatch(const moe_dims &d, int T, const void *x,
                                        const void *w_router, int32_t *idx, float *gate,
                                        int32_t *counts, int32_t *offsets, int32_t *perm,
                                        int32_t *inv_perm, cudaStream_t st);
cudaError_t launch_layer_dispatch(const moe_dims &d, int T, const int32_t *idx, int32_t *counts,
                                  int32_t *offsets, int32_t *perm, int32_t *inv_perm,
                                  cudaStream_t st);
cudaError_t launch_layer_combine(const moe_dims &d, int T, const float *y, const int32_t *inv_perm,
                                 const float *gate, const void *residual, void *out,
                                 cudaStream_t st);

}  // namespace moe
