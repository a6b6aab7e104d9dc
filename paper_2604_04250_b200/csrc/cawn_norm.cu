// Group norm with an activation: entry points, groups too wide for a team of lanes, parameter sums.
#include "cawn_norm.cuh"

namespace cawn {
namespace {

__device__ __forceinline__ float wide_act_backward(int act, float dy, float z, float &g)
{
    return act == CAWN_NORM_ACT_SILU ? act_backward<CAWN_NORM_ACT_SILU>(dy, z, g)
           : act == CAWN_NORM_ACT_GATE ? act_backward<CAWN_NORM_ACT_GATE>(dy, z, g) : dy;
}

// Groups that a team cannot hold in registers: a block per group and stretch of rows, re-reading the
// row from cache for each pass.  Column sums live in shared memory (2 M floats, M <= 4096).
constexpr int kWideThreads = 256;

__device__ __forceinline__ float block_sum(float v, float *red)
{
    v = team_sum<32>(v);
    __syncthreads();
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
    __syncthreads();
    float s = 0.f;
    for (int i = 0; i < kWideThreads / 32; i++) s += red[i];
    return s;
}

template <class T, bool BWD>
__global__ void __launch_bounds__(kWideThreads) norm_wide_kernel(const NormParams P)
{
    follow_previous();
    __shared__ float red[kWideThreads / 32];
    extern __shared__ float fold[];
    const int c0 = blockIdx.y * P.M;
    const long long r0 = (long long)blockIdx.x * P.rows_per_block;
    const long long r1 = r0 + P.rows_per_block < P.N ? r0 + P.rows_per_block : P.N;
    if (BWD && P.part != nullptr)
        for (int i = threadIdx.x; i < 2 * P.M; i += kWideThreads) fold[i] = 0.f;   // each thread its own columns
    for (long long r = r0; r < r1; r++) {
        const T *x = static_cast<const T *>(P.x) + r * P.x_stride + c0;
        const T *gate = P.act == CAWN_NORM_ACT_GATE ? static_cast<const T *>(P.gate) + r * P.gate_stride + c0 : nullptr;
        float s = 0.f, q = 0.f;
        if (!P.rms)
            for (int i = threadIdx.x; i < P.M; i += kWideThreads) s += widen(x[i]);
        const float mean = P.rms ? 0.f : block_sum(s, red) * P.inv_m;
        for (int i = threadIdx.x; i < P.M; i += kWideThreads) {
            const float v = widen(x[i]) - mean;
            q += v * v;
        }
        const float rstd = rsqrtf(block_sum(q, red) * P.inv_m + P.eps);
        float s1 = 0.f, s2 = 0.f;
        for (int pass = 0; pass < (BWD ? 2 : 1); pass++) {
            for (int i = threadIdx.x; i < P.M; i += kWideThreads) {
                const float xh = (widen(x[i]) - mean) * rstd;
                const float wt = P.w != nullptr ? P.w[c0 + i] : 1.f, z = fmaf(xh, wt, P.b != nullptr ? P.b[c0 + i] : 0.f);
                float g = gate != nullptr ? widen(gate[i]) : 0.f;
                if constexpr (!BWD) {
                    float y = z;
                    if (P.act == CAWN_NORM_ACT_SILU) y *= sigmoidf(z);
                    if (P.act == CAWN_NORM_ACT_GATE) y *= g * sigmoidf(g);
                    static_cast<T *>(P.y)[r * P.C + c0 + i] = narrow<T>(y);
                } else {
                    const float dz = wide_act_backward(P.act, widen(static_cast<const T *>(P.gy)[r * P.C + c0 + i]), z, g);
                    if (pass == 0) {
                        s1 += dz * wt;
                        s2 += dz * wt * xh;
                    } else {
                        if (P.part != nullptr) {
                            fold[i] += dz * xh;
                            fold[P.M + i] += dz;
                        }
                        static_cast<T *>(P.gx)[r * P.C + c0 + i] = narrow<T>(rstd * (dz * wt - s1 - xh * s2));
                        if (gate != nullptr) static_cast<T *>(P.ggate)[r * P.C + c0 + i] = narrow<T>(g);
                    }
                }
            }
            if (BWD && pass == 0) {
                s2 = block_sum(s2, red) * P.inv_m;
                s1 = P.rms ? 0.f : block_sum(s1, red) * P.inv_m;
            }
        }
    }
    if (BWD && P.part != nullptr) {
        float *pw = P.part + (size_t)blockIdx.x * 2 * P.C + c0;
        for (int i = threadIdx.x; i < P.M; i += kWideThreads) {
            pw[i] = fold[i];
            pw[P.C + i] = fold[P.M + i];
        }
    }
}

// Parameter gradients: 32 columns a block, 32 row lanes with two sums each, doubles, fixed order.
__global__ void __launch_bounds__(1024) norm_sum_kernel(const float *part, int blocks, int C, float *gw, float *gb)
{
    follow_previous();
    __shared__ double sums[32][33];
    const int x = threadIdx.x % 32, lane = threadIdx.x / 32, col = blockIdx.x * 32 + x;
    double s = 0.0, t = 0.0;
    if (col < 2 * C) {
        int i = lane;
        for (; i + 32 < blocks; i += 64) {
            s += (double)part[(size_t)i * 2 * C + col];
            t += (double)part[(size_t)(i + 32) * 2 * C + col];
        }
        if (i < blocks) s += (double)part[(size_t)i * 2 * C + col];
    }
    sums[lane][x] = s + t;
    __syncthreads();
    // a warp per column: lane x holds row lane x of column `lane`
    s = sums[x][lane];
#pragma unroll
    for (int o = 16; o > 0; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int mine = blockIdx.x * 32 + lane;
    if (x == 0 && mine < 2 * C) {
        if (mine < C) {
            if (gw != nullptr) gw[mine] = (float)s;
        } else if (gb != nullptr) {
            gb[mine - C] = (float)s;
        }
    }
}

int check(const cawn_norm_params *p)
{
    if (p == nullptr) return CAWN_ERR_NULL_POINTER;
    if (p->struct_size != sizeof(cawn_norm_params)) return CAWN_ERR_INVALID_ARG;
    if (p->N < 0 || p->G < 1 || p->M < 1 || !(p->eps >= 0.f) || p->reserved != 0 || !storage_flags_ok(p->flags) ||
        p->act < CAWN_NORM_ACT_NONE || p->act > CAWN_NORM_ACT_GATE || (p->rms != 0 && p->rms != 1))
        return CAWN_ERR_INVALID_ARG;
    const int64_t C = (int64_t)p->G * p->M;
    if ((p->x_stride != 0 && p->x_stride < C) || (p->gate_stride != 0 && p->gate_stride < C)) return CAWN_ERR_INVALID_ARG;
    if (p->M > 4096 || C > (1 << 24) || p->G > 65535) return CAWN_ERR_UNSUPPORTED;
    const int64_t wide = p->x_stride > p->gate_stride ? p->x_stride : p->gate_stride;
    if ((double)p->N * (double)(wide > C ? wide : C) > 1.0e17 || p->N > ((int64_t)1 << 32)) return CAWN_ERR_UNSUPPORTED;
    return CAWN_OK;
}

NormParams fill(const cawn_norm_params *p, const Cut &c)
{
    NormParams P = {};
    P.N = p->N; P.G = p->G; P.M = p->M; P.C = p->G * p->M; P.act = p->act;
    P.x_stride = p->x_stride != 0 ? p->x_stride : P.C;
    P.gate_stride = p->gate_stride != 0 ? p->gate_stride : P.C;
    P.TX = c.TX; P.TY = c.TY; P.rows_per_block = c.rows;
    P.eps = p->eps; P.inv_m = 1.f / (float)p->M; P.rms = p->rms != 0;
    return P;
}

int run(const cawn_norm_params *p, const Cut &c, const NormParams &P, bool bwd, cudaStream_t st)
{
    const bool half = p->flags != 0, sums = bwd && P.part != nullptr;
    if (c.lpg == 0) {
        NormKernel k = half ? (bwd ? norm_wide_kernel<bf16, true> : norm_wide_kernel<bf16, false>)
                            : (bwd ? norm_wide_kernel<float, true> : norm_wide_kernel<float, false>);
        return status_of(launch<true>(k, dim3(c.bx, c.by), dim3(kWideThreads), sums ? (size_t)2 * P.M * sizeof(float) : 0, st, P));
    }
    NormKernel k = bwd ? norm_bwd_pick(c, half, p->act) : norm_fwd_pick(c, half, p->act);
    const size_t fold = sums ? (size_t)2 * c.TX * c.nv * c.v * sizeof(float) : 0;     // up to 64 KB: 256 slots of 32 channels
    if (fold > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)fold);
        if (e != cudaSuccess) return status_of(e);
    }
    return status_of(launch<true>(k, dim3(c.bx, c.by), dim3(threads_of(c)), fold, st, P));
}

}  // namespace
}  // namespace cawn

extern "C" int cawn_group_norm_fwd(const cawn_norm_params *params, const void *x, const float *weight, const float *bias,
                                   const void *gate, void *y, void *cuda_stream)
{
    using namespace cawn;
    const int rc = check(params);
    if (rc != CAWN_OK) return rc;
    if (params->N == 0) return CAWN_OK;
    if (x == nullptr || y == nullptr || (params->act == CAWN_NORM_ACT_GATE && gate == nullptr)) return CAWN_ERR_NULL_POINTER;
    if (!all_aligned16(x, weight, bias, gate, y)) return CAWN_ERR_MISALIGNED;
    const Cut c = cut_of(params, false);
    NormParams P = fill(params, c);
    P.x = x; P.w = weight; P.b = bias; P.gate = gate; P.y = y;
    return run(params, c, P, false, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int cawn_group_norm_workspace_bytes(const cawn_norm_params *params, size_t *bytes)
{
    using namespace cawn;
    const int rc = check(params);
    if (rc != CAWN_OK) return rc;
    if (bytes == nullptr) return CAWN_ERR_NULL_POINTER;
    *bytes = (size_t)cut_of(params, true).most * 2 * params->G * params->M * sizeof(float);
    return CAWN_OK;
}

extern "C" int cawn_group_norm_bwd(const cawn_norm_params *params, const void *x, const float *weight, const float *bias,
                                   const void *gate, const void *grad_y, void *grad_x, void *grad_gate, float *grad_weight,
                                   float *grad_bias, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    using namespace cawn;
    const int rc = check(params);
    if (rc != CAWN_OK) return rc;
    const bool gated = params->act == CAWN_NORM_ACT_GATE, sums = grad_weight != nullptr || grad_bias != nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const Cut c = cut_of(params, true);
    const int C = params->G * params->M;
    if (params->N > 0 && (x == nullptr || grad_y == nullptr || grad_x == nullptr || (gated && (gate == nullptr || grad_gate == nullptr))))
        return CAWN_ERR_NULL_POINTER;
    if (!gated && grad_gate != nullptr) return CAWN_ERR_INVALID_ARG;
    if (sums && workspace == nullptr) return CAWN_ERR_NULL_POINTER;
    if (!all_aligned16(x, weight, bias, gate, grad_y, grad_x, grad_gate, grad_weight, grad_bias, workspace)) return CAWN_ERR_MISALIGNED;
    if (sums && workspace_bytes < (size_t)c.bx * 2 * C * sizeof(float)) return CAWN_ERR_WORKSPACE_TOO_SMALL;
    if (params->N == 0) {
        if (grad_weight != nullptr && cudaMemsetAsync(grad_weight, 0, (size_t)C * sizeof(float), st) != cudaSuccess) return CAWN_ERR_CUDA;
        if (grad_bias != nullptr && cudaMemsetAsync(grad_bias, 0, (size_t)C * sizeof(float), st) != cudaSuccess) return CAWN_ERR_CUDA;
        return CAWN_OK;
    }
    NormParams P = fill(params, c);
    P.x = x; P.w = weight; P.b = bias; P.gate = gate; P.gy = grad_y; P.gx = grad_x; P.ggate = grad_gate;
    P.part = sums ? static_cast<float *>(workspace) : nullptr;
    const int first = run(params, c, P, true, st);
    if (first != CAWN_OK || !sums) return first;
    return status_of(launch<true>(norm_sum_kernel, dim3((2 * C + 31) / 32), dim3(1024), 0, st, (const float *)P.part, c.bx, C, grad_weight, grad_bias));
}
