// gate.cuh -- launchers of the experts' choice (gate.cu) and of the parts of the router that it shares with
// vmoe_route (route.cu) and vmoe_router_bwd (router_bwd.cu) (internal).
#pragma once

#include "common.cuh"

namespace vmoe {

struct Gating {
    int score, groups, kept, top;
    float scale;
    bool renorm;
};

size_t gate_workspace(const Dims &p);
int launch_gate(const Dims &p, const Gating &g, const float *logits, const float *sbias, const uint8_t *mask, int32_t *idx,
                float *gate, int32_t *slot, int32_t *load, int32_t *demand, int32_t *hist, cudaStream_t s);
int launch_gate_grad(const Dims &p, const Gating &g, const float *logits, const int32_t *idx, const float *gate,
                     const int32_t *slot, const void *dy, const void *ye, float *dgate, float *dlogits, cudaStream_t s);
int launch_gate_grad_dx(const Dims &p, const Gating &g, const float *wr, const float *logits, const int32_t *idx,
                        const float *gate, const int32_t *slot, const void *dy, const void *ye, float *dgate, float *dlogits,
                        const void *dx_in, void *dx, cudaStream_t s);
int launch_gate_bias(const Dims &p, const int32_t *demand, float rate, float *bias, cudaStream_t s);

// The router's logits alone.
int launch_router_logits(const Dims &p, const void *x, const float *w_router, const float *bias, float *logits,
                         cudaStream_t s);
// dX = dX_in + dlogits W_r^T (dX_in may be dX), then dW_r and dbias.
int launch_router_grads(const Dims &p, const void *x, const float *w_router, const float *dlogits, float *dw_router,
                        float *dbias, const void *dx_in, void *dx, cudaStream_t s);

}  // namespace vmoe
