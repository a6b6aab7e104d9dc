// Gated delta rule: what its translation units share.
#pragma once
#include "cawn_ops.cuh"

namespace cawn {

struct DeltaParams {
    const void *q, *k, *v;
    const float *g, *beta, *state_in;
    void *o;
    float *state_out;
    long long L, q_stride, k_stride, v_stride, o_stride;     // strides in elements, from step to step
    int B, Hk, Hv, Dk, Dv;
    float scale;
};

// e^g of a log decay; everything below e^-104 is zero in float.
__device__ __forceinline__ float decay_of(float g) { return __expf(g); }

cudaError_t launch_delta_step(const DeltaParams &P, bool half, cudaStream_t st);

}  // namespace cawn
