// Group norm with an activation: forward kernels of the groups that a team of lanes holds.
#include "cawn_norm.cuh"

namespace cawn {
namespace {

template <class T, int LPG, int V, int NV, int ACT>
__global__ void __launch_bounds__(kNormThreads) norm_fwd_kernel(const NormParams P)
{
    follow_previous();
    using U = typename UnitOf<V>::type;
    constexpr int N = UnitOf<V>::N;
    constexpr bool GATED = ACT == CAWN_NORM_ACT_GATE;
    int ch[NV];
    const int ty = my_place<LPG, V>(P, ch);
    U w[NV][N], b[NV][N];
#pragma unroll
    for (int j = 0; j < NV; j++) {
        load_units<V>(w[j], ch[j] >= 0 && P.w != nullptr ? P.w + ch[j] : nullptr, 1.f);
        load_units<V>(b[j], ch[j] >= 0 && P.b != nullptr ? P.b + ch[j] : nullptr, 0.f);
    }
    const long long r0 = (long long)blockIdx.x * P.rows_per_block;
    const long long r1 = r0 + P.rows_per_block < P.N ? r0 + P.rows_per_block : P.N;
    // the bound is the block's, not the row's: whole warps stay in the loop for the shuffles
    for (long long base = r0; base < r1; base += P.TY) {
        const long long r = base + ty;
        const bool live = r < r1 && ty < P.TY;
        Word<T, V> xw[NV], gw[NV];
        U f[NV][N], g[NV][N];
#pragma unroll
        for (int j = 0; j < NV; j++)
            if (live && ch[j] >= 0) {
                xw[j].get(static_cast<const T *>(P.x) + r * P.x_stride + ch[j]);
                if (GATED) gw[j].get(static_cast<const T *>(P.gate) + r * P.gate_stride + ch[j]);
            }
#pragma unroll
        for (int j = 0; j < NV; j++) {
#pragma unroll
            for (int i = 0; i < N; i++) { f[j][i] = both<U>(0.f); g[j][i] = both<U>(0.f); }
            if (live && ch[j] >= 0) {
                xw[j].to(f[j]);
                if (GATED) gw[j].to(g[j]);
            }
        }
        normalise<LPG>(f, ch, P);
#pragma unroll
        for (int j = 0; j < NV; j++) {
            if (!live || ch[j] < 0) continue;
#pragma unroll
            for (int i = 0; i < N; i++) {
                U z = fma2(f[j][i], w[j][i], b[j][i]);
                if (ACT == CAWN_NORM_ACT_SILU) z = mul2(z, sigmoid2(z));
                if (GATED) z = mul2(z, mul2(g[j][i], sigmoid2(g[j][i])));
                f[j][i] = z;
            }
            xw[j].from(f[j]);
            xw[j].put(static_cast<T *>(P.y) + r * P.C + ch[j]);
        }
    }
}

template <class T, int V, int ACT> NormKernel of_cut(const Cut &c)
{
    if (c.lpg == 4) return norm_fwd_kernel<T, 4, V, 1, ACT>;
    if (c.lpg == 8) return norm_fwd_kernel<T, 8, V, 1, ACT>;
    if (c.lpg == 16) return norm_fwd_kernel<T, 16, V, 1, ACT>;
    if (c.nv == 1) return norm_fwd_kernel<T, 32, V, 1, ACT>;
    if (c.nv == 2) return norm_fwd_kernel<T, 32, V, 2, ACT>;
    if constexpr (V == 8) return norm_fwd_kernel<T, 32, V, 4, ACT>;
    else return c.nv == 4 ? norm_fwd_kernel<T, 32, V, 4, ACT> : norm_fwd_kernel<T, 32, V, 8, ACT>;
}
template <class T> NormKernel of_act(const Cut &c, int act)
{
    constexpr int W = 16 / (int)sizeof(T);
    if (act == CAWN_NORM_ACT_SILU) return c.v == 1 ? of_cut<T, 1, CAWN_NORM_ACT_SILU>(c) : of_cut<T, W, CAWN_NORM_ACT_SILU>(c);
    if (act == CAWN_NORM_ACT_GATE) return c.v == 1 ? of_cut<T, 1, CAWN_NORM_ACT_GATE>(c) : of_cut<T, W, CAWN_NORM_ACT_GATE>(c);
    return c.v == 1 ? of_cut<T, 1, CAWN_NORM_ACT_NONE>(c) : of_cut<T, W, CAWN_NORM_ACT_NONE>(c);
}

}  // namespace

NormKernel norm_fwd_pick(const Cut &c, bool half, int act) { return half ? of_act<bf16>(c, act) : of_act<float>(c, act); }

}  // namespace cawn
