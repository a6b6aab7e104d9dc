// Selective scan, token by token, for decoding.
//
// Mathematics: see cawn_selective.cuh; a few tokens with the state in registers.
// Bound: the state is read and written once (8 bytes a cell), everything else is a few numbers a channel.  A lane has four
// neighbouring states of a channel, so a warp's accesses to the states are whole lines; lanes of a channel read the same
// x, dt and z.
#include "cawn_selective.cuh"

namespace cawn {
namespace {

constexpr int kStepThreads = 128;

template <class T, int NL>          // lanes a channel
__global__ void __launch_bounds__(kStepThreads) selective_step_kernel(const SelectiveParams P)
{
    follow_previous();
    const long long at = ((long long)blockIdx.x * kStepThreads + threadIdx.x) / NL;        // b * D + c
    const int n0 = threadIdx.x % NL * 4;
    const bool in = at < (long long)P.seq.B * P.D;
    const int b = in ? (int)(at / P.D) : 0, c = in ? (int)(at % P.D) : 0, g = c / P.Dg;
    f32x2 A2[2], h[2];
    load_states<4>(A2, P.A + (long long)c * P.N, n0, P.N, in);
    load_states<4>(h, P.state_in + at * P.N, n0, P.N, in && P.state_in != nullptr);
    A2[0] = mul2(A2[0], twice(kLog2e));
    A2[1] = mul2(A2[1], twice(kLog2e));
    const float bias = P.dt_bias != nullptr ? P.dt_bias[c] : 0.f, skip = P.skip != nullptr ? P.skip[c] : 0.f;
    for (long long t = 0; t < P.seq.L; t++) {
        const long long row = b * P.seq.L + t;
        const float x = widen(static_cast<const T *>(P.x)[row * P.xs + c]), raw = widen(static_cast<const T *>(P.dt)[row * P.dts + c]) + bias;
        const float z = P.z != nullptr ? widen(static_cast<const T *>(P.z)[row * P.zs + c]) : 0.f;
        const float4 B = fetch_quad(static_cast<const T *>(P.bm) + row * P.bs + g * P.N + n0, P.N - n0, P.whole_b).get();
        const float4 C = fetch_quad(static_cast<const T *>(P.cm) + row * P.cs + g * P.N + n0, P.N - n0, P.whole_c).get();
        const float d = P.softplus ? softplus_of(raw) : raw;
        const f32x2 dl = twice(d), dx = twice(d * x);
        h[0] = fma2(exp2_pair(mul2(dl, A2[0])), h[0], mul2(dx, pair(B.x, B.y)));
        h[1] = fma2(exp2_pair(mul2(dl, A2[1])), h[1], mul2(dx, pair(B.z, B.w)));
        float v = sum_of(fma2(h[1], pair(C.z, C.w), mul2(h[0], pair(C.x, C.y))));
#pragma unroll
        for (int o = NL / 2; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
        v = fmaf(skip, x, v);
        if (P.z != nullptr) v *= z * sigmoid_of(z);
        if (in && n0 == 0) static_cast<T *>(P.y)[row * P.D + c] = narrow<T>(v);
    }
    if (P.state_out != nullptr) store_states<4>(P.state_out + at * P.N, h, n0, P.N, in);
}

template <class T> SelectiveKernel pick(int nl)
{
    return nl == 1 ? selective_step_kernel<T, 1> : nl == 2 ? selective_step_kernel<T, 2> : nl == 4 ? selective_step_kernel<T, 4>
           : nl == 8 ? selective_step_kernel<T, 8> : selective_step_kernel<T, 16>;
}

}  // namespace

int launch_selective_step(const SelectiveParams &P, bool half, cudaStream_t st)
{
    const int nl = P.N <= 4 ? 1 : P.N <= 8 ? 2 : P.N <= 16 ? 4 : P.N <= 32 ? 8 : 16;
    const long long blocks = ceil_div((int64_t)P.seq.B * P.D * nl, kStepThreads);
    return status_of(launch<true>(half ? pick<bf16>(nl) : pick<float>(nl), dim3((unsigned)blocks), dim3(kStepThreads), 0, st, P));
}

}  // namespace cawn
