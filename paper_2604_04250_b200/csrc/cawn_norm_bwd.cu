// Group norm with an activation: backward kernels of the groups that a team of lanes holds.
//
// Parameter gradients are register sums of a thread's channels over the rows it walks; they are folded per block in
// shared memory, written as one partial row per block, and summed in double in a fixed order by a second launch.
#include "cawn_norm.cuh"

namespace cawn {
namespace {

template <class T, int LPG, int V, int NV, int ACT>
__global__ void __launch_bounds__(kNormThreads) norm_bwd_kernel(const NormParams P)
{
    follow_previous();
    using U = typename UnitOf<V>::type;
    constexpr int N = UnitOf<V>::N;
    constexpr bool GATED = ACT == CAWN_NORM_ACT_GATE;
    constexpr bool KEEP = NV * V <= 16;             // weights stay in registers; more come from L1 row by row
    extern __shared__ float fold[];                 // [2][TX * NV * V]
    int ch[NV];
    const int ty = my_place<LPG, V>(P, ch), tx = threadIdx.x % P.TX, TY = P.TY;
    U w[KEEP ? NV : 1][N], b[KEEP ? NV : 1][N], sw[NV][N], sb[NV][N];
    auto weights = [&](int j, U (&wt)[N], U (&bt)[N]) {
        load_units<V>(wt, ch[j] >= 0 && P.w != nullptr ? P.w + ch[j] : nullptr, 1.f);
        load_units<V>(bt, ch[j] >= 0 && P.b != nullptr ? P.b + ch[j] : nullptr, 0.f);
    };
#pragma unroll
    for (int j = 0; j < NV; j++) {
        if constexpr (KEEP) weights(j, w[j], b[j]);
#pragma unroll
        for (int i = 0; i < N; i++) { sw[j][i] = both<U>(0.f); sb[j][i] = both<U>(0.f); }
    }
    const long long r0 = (long long)blockIdx.x * P.rows_per_block;
    const long long r1 = r0 + P.rows_per_block < P.N ? r0 + P.rows_per_block : P.N;
    Word<T, V> xw[NV], dw[NV], gw[NV];
    auto fetch = [&](long long r) {
#pragma unroll
        for (int j = 0; j < NV; j++)
            if (r < r1 && ty < TY && ch[j] >= 0) {
                xw[j].get(static_cast<const T *>(P.x) + r * P.x_stride + ch[j]);
                dw[j].get(static_cast<const T *>(P.gy) + r * P.C + ch[j]);
                if (GATED) gw[j].get(static_cast<const T *>(P.gate) + r * P.gate_stride + ch[j]);
            }
    };
    fetch(r0 + ty);
    // the bound is the block's, not the row's: whole warps stay in the loop for the shuffles
    for (long long base = r0; base < r1; base += TY) {
        const long long r = base + ty;
        const bool live = r < r1 && ty < TY;
        U f[NV][N], d[NV][N], g[NV][N];
#pragma unroll
        for (int j = 0; j < NV; j++) {
#pragma unroll
            for (int i = 0; i < N; i++) { f[j][i] = both<U>(0.f); d[j][i] = both<U>(0.f); g[j][i] = both<U>(0.f); }
            if (live && ch[j] >= 0) {
                xw[j].to(f[j]);
                dw[j].to(d[j]);
                if (GATED) gw[j].to(g[j]);
            }
        }
        fetch(r + TY);                  // the next row, while this one is worked on
        const float rstd = normalise<LPG>(f, ch, P);
        U u1 = both<U>(0.f), u2 = both<U>(0.f);
#pragma unroll
        for (int j = 0; j < NV; j++) {
            if constexpr (!KEEP) weights(j, w[0], b[0]);
            const int k = KEEP ? j : 0;
#pragma unroll
            for (int i = 0; i < N && live; i++) {       // words past the group's end: d = 0, and all sums get 0
                const U dz = act_backward<ACT>(d[j][i], fma2(f[j][i], w[k][i], b[k][i]), g[j][i]);
                sw[j][i] = fma2(dz, f[j][i], sw[j][i]);
                sb[j][i] = add2(sb[j][i], dz);
                d[j][i] = mul2(dz, w[k][i]);
                u1 = add2(u1, d[j][i]);
                u2 = fma2(d[j][i], f[j][i], u2);
            }
        }
        const U s2 = both<U>(-team_sum<LPG>(total(u2)) * P.inv_m), s1 = both<U>(P.rms ? 0.f : -team_sum<LPG>(total(u1)) * P.inv_m), rs = both<U>(rstd);
#pragma unroll
        for (int j = 0; j < NV; j++) {
            if (!live || ch[j] < 0) continue;
#pragma unroll
            for (int i = 0; i < N; i++) d[j][i] = mul2(rs, fma2(f[j][i], s2, add2(d[j][i], s1)));
            Word<T, V> out;
            out.from(d[j]);
            out.put(static_cast<T *>(P.gx) + r * P.C + ch[j]);
            if (GATED) {
                out.from(g[j]);
                out.put(static_cast<T *>(P.ggate) + r * P.C + ch[j]);
            }
        }
    }
    if (P.part == nullptr) return;
    // row lanes fold their sums one after the other in a fixed order: shared memory holds one row
    const int half = NV * V * P.TX;
    for (int turn = 0; turn < TY; turn++) {
        if (ty == turn) {
#pragma unroll
            for (int j = 0; j < NV; j++)
#pragma unroll
                for (int i = 0; i < N; i++) {
                    const float *a = reinterpret_cast<const float *>(&sw[j][i]), *c = reinterpret_cast<const float *>(&sb[j][i]);
#pragma unroll
                    for (int e = 0; e < V / N; e++) {
                        const int at = (j * V + i * (V / N) + e) * P.TX + tx;
                        fold[at] = turn == 0 ? a[e] : fold[at] + a[e];
                        fold[half + at] = turn == 0 ? c[e] : fold[half + at] + c[e];
                    }
                }
        }
        __syncthreads();
    }
    if (ty == 0) {
        float *pw = P.part + (size_t)blockIdx.x * 2 * P.C;
#pragma unroll
        for (int j = 0; j < NV; j++)
            if (ch[j] >= 0)
#pragma unroll
                for (int e = 0; e < V; e++) {
                    const int at = (j * V + e) * P.TX + tx;
                    pw[ch[j] + e] = fold[at];
                    pw[P.C + ch[j] + e] = fold[half + at];
                }
    }
}

template <class T, int V, int ACT> NormKernel of_cut(const Cut &c)
{
    if (c.lpg == 4) return norm_bwd_kernel<T, 4, V, 1, ACT>;
    if (c.lpg == 8) return norm_bwd_kernel<T, 8, V, 1, ACT>;
    if (c.lpg == 16) return norm_bwd_kernel<T, 16, V, 1, ACT>;
    if (c.nv == 1) return norm_bwd_kernel<T, 32, V, 1, ACT>;
    if (c.nv == 2) return norm_bwd_kernel<T, 32, V, 2, ACT>;
    if constexpr (V == 8) return norm_bwd_kernel<T, 32, V, 4, ACT>;
    else return c.nv == 4 ? norm_bwd_kernel<T, 32, V, 4, ACT> : norm_bwd_kernel<T, 32, V, 8, ACT>;
}
template <class T> NormKernel of_act(const Cut &c, int act)
{
    constexpr int W = 16 / (int)sizeof(T);
    if (act == CAWN_NORM_ACT_SILU) return c.v == 1 ? of_cut<T, 1, CAWN_NORM_ACT_SILU>(c) : of_cut<T, W, CAWN_NORM_ACT_SILU>(c);
    if (act == CAWN_NORM_ACT_GATE) return c.v == 1 ? of_cut<T, 1, CAWN_NORM_ACT_GATE>(c) : of_cut<T, W, CAWN_NORM_ACT_GATE>(c);
    return c.v == 1 ? of_cut<T, 1, CAWN_NORM_ACT_NONE>(c) : of_cut<T, W, CAWN_NORM_ACT_NONE>(c);
}

}  // namespace

NormKernel norm_bwd_pick(const Cut &c, bool half, int act) { return half ? of_act<bf16>(c, act) : of_act<float>(c, act); }

}  // namespace cawn
