// Gated delta rule, token by token.
//
// Mathematics, per value row (a Dk-vector s of the state): s <- a s, u = beta (v - s.k), s <- s + u k,
// o = scale s.q.  With both dot products taken on the old row, s.k and s.q, the new row's read-out is
// a s.q + u k.q, so one reduction round serves both.
// Bound: the state is read and written once (8 bytes a cell), everything else is Dk + Dv numbers; a
// call is HBM-bound for a batch and latency-bound for one stream.  A row is dealt to LPR lanes, 8 floats
// each as two float4 (coalesced, no shared memory); a thread holds R rows so that a batch keeps R * 32
// bytes per thread in flight, while few rows take R = 1 and spread over more SMs.
#include "cawn_delta.cuh"

namespace cawn {
namespace {

constexpr int kStepThreads = 128;

template <class T, int LPR, int R>
__global__ void __launch_bounds__(kStepThreads) delta_step_kernel(const DeltaParams P)
{
    constexpr int kRowsWarp = 32 / LPR, kRowsPass = kStepThreads / LPR;
    const int lane = threadIdx.x % LPR, row0 = blockIdx.y * (kRowsPass * R) + (threadIdx.x / 32) * kRowsWarp + (threadIdx.x % 32) / LPR;
    const int bh = blockIdx.x, b = bh / P.Hv, h = bh % P.Hv, hk = h / (P.Hv / P.Hk);
    const int c0 = lane * 4, c1 = (LPR + lane) * 4;              // this lane's columns: c0..c0+3 and c1..c1+3
    const bool in0 = c0 < P.Dk, in1 = c1 < P.Dk;
    const long long srow = (long long)bh * P.Dv * P.Dk;
    const T *q = static_cast<const T *>(P.q) + (long long)b * P.L * P.q_stride + (long long)hk * P.Dk;
    const T *k = static_cast<const T *>(P.k) + (long long)b * P.L * P.k_stride + (long long)hk * P.Dk;
    const T *v = static_cast<const T *>(P.v) + (long long)b * P.L * P.v_stride + (long long)h * P.Dv;
    T *o = static_cast<T *>(P.o) + (long long)b * P.L * P.o_stride + (long long)h * P.Dv;
    const float *g = P.g + (long long)b * P.L * P.Hv + h, *beta = P.beta + (long long)b * P.L * P.Hv + h;

    float s[R][8];
    int row[R];
#pragma unroll
    for (int i = 0; i < R; i++) {
        row[i] = row0 + i * kRowsPass;
        float4 lo = make_float4(0.f, 0.f, 0.f, 0.f), hi = lo;
        if (P.state_in != nullptr && row[i] < P.Dv) {
            const float *src = P.state_in + srow + (long long)row[i] * P.Dk;
            if (in0) lo = *reinterpret_cast<const float4 *>(src + c0);
            if (in1) hi = *reinterpret_cast<const float4 *>(src + c1);
        }
        s[i][0] = lo.x; s[i][1] = lo.y; s[i][2] = lo.z; s[i][3] = lo.w;
        s[i][4] = hi.x; s[i][5] = hi.y; s[i][6] = hi.z; s[i][7] = hi.w;
    }
    for (long long t = 0; t < P.L; t++) {
        float kv[8], qv[8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const int c = e < 4 ? c0 + e : c1 + e - 4;
            const bool in = e < 4 ? in0 : in1;
            kv[e] = in ? widen(k[t * P.k_stride + c]) : 0.f;
            qv[e] = in ? widen(q[t * P.q_stride + c]) : 0.f;
        }
        const float a = decay_of(g[t * P.Hv]), bt = beta[t * P.Hv];
        float vv[R];
#pragma unroll
        for (int i = 0; i < R; i++) vv[i] = row[i] < P.Dv ? widen(v[t * P.v_stride + row[i]]) : 0.f;
        float kq = 0.f, sk[R], sq[R];
#pragma unroll
        for (int e = 0; e < 8; e++) kq = fmaf(kv[e], qv[e], kq);
#pragma unroll
        for (int i = 0; i < R; i++) {
            sk[i] = 0.f; sq[i] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                sk[i] = fmaf(s[i][e], kv[e], sk[i]);
                sq[i] = fmaf(s[i][e], qv[e], sq[i]);
            }
        }
#pragma unroll
        for (int m = LPR / 2; m > 0; m /= 2) {
            kq += __shfl_xor_sync(0xffffffffu, kq, m);
#pragma unroll
            for (int i = 0; i < R; i++) {
                sk[i] += __shfl_xor_sync(0xffffffffu, sk[i], m);
                sq[i] += __shfl_xor_sync(0xffffffffu, sq[i], m);
            }
        }
#pragma unroll
        for (int i = 0; i < R; i++) {
            const float u = bt * (vv[i] - a * sk[i]);
#pragma unroll
            for (int e = 0; e < 8; e++) s[i][e] = fmaf(u, kv[e], a * s[i][e]);
            if (lane == 0 && row[i] < P.Dv) o[t * P.o_stride + row[i]] = narrow<T>(P.scale * fmaf(u, kq, a * sq[i]));
        }
    }
    if (P.state_out == nullptr) return;
#pragma unroll
    for (int i = 0; i < R; i++) {
        if (row[i] >= P.Dv) continue;
        float *dst = P.state_out + srow + (long long)row[i] * P.Dk;
        if (in0) *reinterpret_cast<float4 *>(dst + c0) = make_float4(s[i][0], s[i][1], s[i][2], s[i][3]);
        if (in1) *reinterpret_cast<float4 *>(dst + c1) = make_float4(s[i][4], s[i][5], s[i][6], s[i][7]);
    }
}

template <class T, int LPR> cudaError_t go(const DeltaParams &P, cudaStream_t st)
{
    constexpr int pass = kStepThreads / LPR;
    const long long heads = (long long)P.B * P.Hv;
    const int blocks1 = (P.Dv + pass - 1) / pass, blocks4 = (P.Dv + 4 * pass - 1) / (4 * pass);
    // four rows a thread when that still gives every SM several blocks
    if (heads * blocks4 >= 4ll * sm_count())
        return launch(delta_step_kernel<T, LPR, 4>, dim3((unsigned)heads, blocks4), dim3(kStepThreads), 0, st, P);
    return launch(delta_step_kernel<T, LPR, 1>, dim3((unsigned)heads, blocks1), dim3(kStepThreads), 0, st, P);
}

}  // namespace

cudaError_t launch_delta_step(const DeltaParams &P, bool half, cudaStream_t st)
{
    // 8 lanes cover 64 columns, 16 lanes 128
    if (P.Dk <= 64) return half ? go<bf16, 8>(P, st) : go<float, 8>(P, st);
    return half ? go<bf16, 16>(P, st) : go<float, 16>(P, st);
}

}  // namespace cawn
