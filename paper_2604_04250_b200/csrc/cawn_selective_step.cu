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

// NL lanes a channel; R sequences a thread.  With R = 4 a lane finds the step and the gate of one sequence and hands them to the
// others, and their sums are scattered back to it, so that they are found once and not by each lane; A is shared
// (256 sequences of 2048 channels of 16, bfloat16: 16 us, memory's time 11; R = 1 30, R = 4 without the handing over 48).
template <class T, int NL, int R, bool WHOLE>
__global__ void __launch_bounds__(kStepThreads) selective_step_kernel(const SelectiveParams P)
{
    follow_previous();
    constexpr unsigned kAll = 0xffffffffu;
    constexpr int Q = R == 1 ? 1 : NL == 1 ? 4 : NL == 2 ? 2 : 1;       // sequences that are this lane's own: nl % 4 + NL q
    // blocks of channels first, then groups of R sequences
    const unsigned across = ((unsigned)P.D * NL + kStepThreads - 1) / kStepThreads, at = (blockIdx.x % across * kStepThreads + threadIdx.x) / NL;
    const int nl = threadIdx.x % NL, n0 = nl * 4, B = P.seq.B;
    const bool there = at < (unsigned)P.D;
    const int c = there ? (int)at : 0, g = P.G == 1 ? 0 : c / P.Dg;
    const long long b0 = (long long)(blockIdx.x / across) * R, L = P.seq.L;
    const int some = B - b0 < R ? (int)(B - b0) : R;                    // sequences that are there
    const long long first = (b0 * P.D + c) * P.N, next = (long long)P.D * P.N;
    const T *bm = static_cast<const T *>(P.bm) + g * P.N + n0, *cm = static_cast<const T *>(P.cm) + g * P.N + n0;
    struct Token { T x[Q], dt[Q], z[Q]; Quad<T> b[R], c[R]; };
    auto token = [&](long long t) {
        Token k;
#pragma unroll
        for (int q = 0; q < Q; q++) {
            const int r = nl % R + NL * q;
            const long long row = (r < some ? b0 + r : b0) * L + t;
            k.x[q] = static_cast<const T *>(P.x)[row * P.xs + c];
            k.dt[q] = static_cast<const T *>(P.dt)[row * P.dts + c];
            k.z[q] = P.z != nullptr ? static_cast<const T *>(P.z)[row * P.zs + c] : narrow<T>(0.f);
        }
#pragma unroll
        for (int r = 0; r < R; r++) {
            const long long row = (r < some ? b0 + r : b0) * L + t;
            k.b[r] = quad_of<WHOLE>(bm + row * P.bs, P.N - n0, P.whole_b);
            k.c[r] = quad_of<WHOLE>(cm + row * P.cs, P.N - n0, P.whole_c);
        }
        return k;
    };
    // everything sets out before anything is waited for
    Quad<float> raw[R];
#pragma unroll
    for (int r = 0; r < R; r++)
        raw[r] = quad_of<WHOLE>(P.state_in + first + r * next + n0, there && r < some && P.state_in != nullptr ? P.N - n0 : 0, P.N % 4 == 0);
    const Quad<float> rawA = quad_of<WHOLE>(P.A + (long long)c * P.N + n0, P.N - n0, P.N % 4 == 0);
    const float bias = P.dt_bias != nullptr ? P.dt_bias[c] : 0.f, skip = P.skip != nullptr ? P.skip[c] : 0.f;
    Token now = {};
    if (L > 0) now = token(0);
    f32x2 A2[2] = {rate_of(pair(rawA.get().x, rawA.get().y)), rate_of(pair(rawA.get().z, rawA.get().w))}, h[R][2];
#pragma unroll
    for (int r = 0; r < R; r++) {
        h[r][0] = pair(raw[r].get().x, raw[r].get().y);
        h[r][1] = pair(raw[r].get().z, raw[r].get().w);
    }
    for (long long t = 0; t < L; t++) {
        float x[Q], d[Q], gate[Q];
#pragma unroll
        for (int q = 0; q < Q; q++) {
            const float in = widen(now.dt[q]) + bias, z = widen(now.z[q]);
            x[q] = widen(now.x[q]);
            d[q] = P.softplus ? softplus_of(in) : in;
            gate[q] = P.z != nullptr ? z * sigmoid_of(z) : 1.f;
        }
        float v[R];
#pragma unroll
        for (int r = 0; r < R; r++) {
            const float4 Bf = now.b[r].get(), Cf = now.c[r].get();
            const int q = R == 1 ? 0 : r / NL < Q ? r / NL : 0;
            const float dr = R == 1 ? d[0] : __shfl_sync(kAll, d[q], r % NL, NL), xr = R == 1 ? x[0] : __shfl_sync(kAll, x[q], r % NL, NL);
            const f32x2 dl = twice(dr), dx = twice(dr * xr);
            h[r][0] = fma2(exp2_pair(mul2(dl, A2[0])), h[r][0], mul2(dx, pair(Bf.x, Bf.y)));
            h[r][1] = fma2(exp2_pair(mul2(dl, A2[1])), h[r][1], mul2(dx, pair(Bf.z, Bf.w)));
            v[r] = sum_of(fma2(h[r][1], pair(Cf.z, Cf.w), mul2(h[r][0], pair(Cf.x, Cf.y))));
        }
        if (t + 1 < L) now = token(t + 1);
        if constexpr (R == 4 && NL >= 2) {      // by halving: each exchange sends half of a lane's sums away and keeps the other half
            const bool odd = nl & 1, high = nl & 2;
            const float a = (odd ? v[1] : v[0]) + __shfl_xor_sync(kAll, odd ? v[0] : v[1], 1);
            const float b = (odd ? v[3] : v[2]) + __shfl_xor_sync(kAll, odd ? v[2] : v[3], 1);
            v[0] = a;
            v[R > 1 ? 1 : 0] = b;
            if constexpr (NL >= 4) v[0] = (high ? b : a) + __shfl_xor_sync(kAll, high ? a : b, 2);
#pragma unroll
            for (int o = 4; o < NL; o *= 2) v[0] += __shfl_xor_sync(kAll, v[0], o);
        } else if constexpr (R == 1) {
#pragma unroll
            for (int o = 1; o < NL; o *= 2) v[0] += __shfl_xor_sync(kAll, v[0], o);
        }
#pragma unroll
        for (int q = 0; q < Q; q++) {
            const int r = nl % R + NL * q;
            if (there && r < some && nl < R) static_cast<T *>(P.y)[((b0 + r) * L + t) * P.D + c] = narrow<T>(fmaf(skip, x[q], v[q]) * gate[q]);
        }
    }
    if (P.state_out != nullptr) {
#pragma unroll
        for (int r = 0; r < R; r++) store_states<4>(P.state_out + first + r * next, h[r], n0, P.N, there && r < some);
    }
}

template <class T, int R, bool WHOLE> SelectiveKernel pick(int nl)
{
    return nl == 1 ? selective_step_kernel<T, 1, R, WHOLE> : nl == 2 ? selective_step_kernel<T, 2, R, WHOLE> : nl == 4 ? selective_step_kernel<T, 4, R, WHOLE>
           : nl == 8 ? selective_step_kernel<T, 8, R, WHOLE> : selective_step_kernel<T, 16, R, WHOLE>;
}
template <class T> SelectiveKernel pick(int nl, bool four, bool whole)
{
    return four ? (whole ? pick<T, 4, true>(nl) : pick<T, 4, false>(nl)) : (whole ? pick<T, 1, true>(nl) : pick<T, 1, false>(nl));
}

}  // namespace

int launch_selective_step(const SelectiveParams &P, bool half, cudaStream_t st)
{
    const int nl = P.N <= 4 ? 1 : P.N <= 8 ? 2 : P.N <= 16 ? 4 : P.N <= 32 ? 8 : 16;
    // four sequences a thread once that leaves 512 threads a multiprocessor
    const bool four = P.seq.B >= 4 && (int64_t)P.seq.B * P.D * nl >= (int64_t)sm_count() * 2048;
    const long long blocks = ceil_div(P.seq.B, four ? 4 : 1) * ceil_div((int64_t)P.D * nl, kStepThreads);
    const bool whole = P.whole_b && P.whole_c;
    const SelectiveKernel k = half ? pick<bf16>(nl, four, whole) : pick<float>(nl, four, whole);
    return status_of(launch<true>(k, dim3((unsigned)blocks), dim3(kStepThreads), 0, st, P));
}

}  // namespace cawn
